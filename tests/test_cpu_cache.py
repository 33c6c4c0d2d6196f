"""CPU checks of the 8-bit cache of keys and values: sizes, the index of a call's rows, and the refusals of the C entry points
(fake pointers, never dereferenced: every call fails, or has nothing to do, before anything is enqueued)."""
import ctypes as C

import numpy as np
import pytest

FAKE = 0x10000


@pytest.fixture(scope="module")
def kv():
    from paper_2605_11222_b200 import build, kvcache
    build.build()
    kvcache._library()
    return kvcache


def _cache(kv, n_pages=4, heads=2, dim=64, page=32, codes=FAKE, scale=FAKE, size=None):
    return kv._Cache(C.sizeof(kv._Cache) if size is None else size, n_pages, heads, dim, page, codes, scale)


def _plan(kv, lengths=(1, 5), group=2, max_pages=3, tables=FAKE, held=FAKE, index=FAKE, size=None):
    p, _ = _filled(kv, lengths, group)
    p.struct_size = C.sizeof(kv._Plan) if size is None else size
    p.max_pages, p.d_tables, p.d_held, p.d_index = max_pages, tables, held, index
    return p


def _filled(kv, lengths, group):
    lib = kv._library()
    lengths = np.asarray(lengths, dtype=np.int64)
    n = lib.admmq_cache_plan_ints(lengths.ctypes.data, len(lengths), group)
    assert n > 0
    index = np.full(n + 4, -7, dtype=np.int32)
    p = kv._Plan(struct_size=C.sizeof(kv._Plan))
    assert lib.admmq_cache_plan_fill(lengths.ctypes.data, len(lengths), group, index.ctypes.data, C.addressof(p)) == 0
    assert (index[n:] == -7).all() and (index[:n] >= 0).all()
    return p, index[:n]


def test_sizes_of_a_cache(kv):
    lib = kv._library()
    assert lib.admmq_cache_code_bytes(10, 8, 128, 64) == 10 * 8 * 64 * 2 * 128
    assert lib.admmq_cache_code_bytes(1, 1, 80, 16) == 16 * 2 * 128          # 80 values: two columns of 64
    assert lib.admmq_cache_scale_bytes(10, 8, 128, 64) == 10 * 8 * 4 * 8
    for bad in [(0, 1, 64, 16), (1, 0, 64, 16), (1, 5000, 64, 16), (1, 1, 8, 16), (1, 1, 72, 16), (1, 1, 272, 16), (1, 1, 64, 8),
                (1, 1, 64, 48), (1, 1, 64, 512), (2 ** 30, 4, 64, 256)]:
        assert lib.admmq_cache_code_bytes(*bad) == 0 and lib.admmq_cache_scale_bytes(*bad) == 0


@pytest.mark.parametrize("lengths,group", [([1], 1), ([1], 16), ([0, 3, 0], 5), ([1, 17, 300, 0, 12, 13], 4), ([5000, 1], 1), ([2], 1024)])
def test_the_index_of_the_rows(kv, lengths, group):
    """Rows, blocks and tiles: every row of every request once, whatever block it begins in."""
    p, index = _filled(kv, lengths, group)
    n = len(lengths)
    pad = lambda k: -(-k // 4) * 4  # noqa: E731
    assert p.n_requests == n and p.group == group and p.n_rows == sum(lengths)
    assert list(index[: n + 1]) == [sum(lengths[:i]) for i in range(n + 1)]
    at = pad(n + 1)
    blocks = index[at: at + 4 * p.n_blocks].reshape(-1, 4)
    assert all(row == sum(lengths[:r]) and n_rows == lengths[r] for r, _, row, n_rows in blocks)
    for i, k in enumerate(lengths):
        mine = sorted(b for r, b, _, _ in blocks if r == i)
        assert mine == list(range((k + 30) // 16 if k else 0))
        for first in range(16):                                      # enough for every place of the first row in its block
            assert k == 0 or (first + k + 15) // 16 <= len(mine)
    at += 4 * p.n_blocks
    small, big = index[at: at + 4 * p.n_small].reshape(-1, 4), index[at + 4 * p.n_small: at + 4 * (p.n_small + p.n_big)].reshape(-1, 4)
    assert len(index) == at + 4 * (p.n_small + p.n_big)
    seen = {i: [] for i in range(n)}
    for tiles, rows in ((small, 16), (big, 256)):
        for request, first, row, length in tiles:
            assert length == lengths[request] and row == sum(lengths[:request]) and first % rows == 0
            seen[request] += range(first, min(first + rows, length * group))
    assert all(sorted(seen[i]) == list(range(lengths[i] * group)) for i in range(n))
    most = [min(16, k * group) for i, k in enumerate(lengths) if i in set(small[:, 0])]
    assert p.small_rows == max(most, default=0)


def test_plans_that_are_refused(kv):
    lib = kv._library()

    def ints(lengths, n, group):
        a = np.asarray(lengths, dtype=np.int64)
        return lib.admmq_cache_plan_ints(a.ctypes.data, n, group)

    assert ints([1], 1, 1) > 0 and ints([0], 1, 1) > 0
    for bad in (([1], 0, 1), ([1], -1, 1), ([-1], 1, 1), ([2 ** 31], 1, 1), ([2 ** 30], 1, 2), ([1], 1, 0), ([1], 1, 1025), ([2 ** 30, 1], 2, 1)):
        assert ints(*bad) == -1
    assert lib.admmq_cache_plan_ints(None, 1, 1) == -1
    p, buf, one = kv._Plan(struct_size=C.sizeof(kv._Plan)), np.zeros(64, np.int32), np.ones(1, np.int64)
    f = lib.admmq_cache_plan_fill
    assert f(one.ctypes.data, 1, 1, None, C.addressof(p)) == 1 and f(one.ctypes.data, 1, 1, buf.ctypes.data, None) == 1
    assert f(one.ctypes.data, 1, 0, buf.ctypes.data, C.addressof(p)) == 2
    p.struct_size -= 4
    assert f(one.ctypes.data, 1, 1, buf.ctypes.data, C.addressof(p)) == 1


@pytest.mark.parametrize("name", ["admmq_cache_write", "admmq_cache_read", "admmq_cache_attend"])
def test_calls_refuse_bad_arguments(kv, name):
    from paper_2605_11222_b200 import binding as B
    f = getattr(kv._library(), name)
    attend = name.endswith("attend")
    ok = ([0.125, 0, FAKE, 256, 64, FAKE, 256, 64, FAKE, FAKE, 0, FAKE, None] if attend
          else [1, FAKE, 128, 64, FAKE, 128, 64, FAKE, None])
    good = _cache(kv), _plan(kv)

    def call(cache=None, plan=None, **kw):
        a = list(ok)
        for i, v in kw.items():
            a[int(i[1:])] = v
        c, p = cache or good[0], plan or good[1]
        return f(C.addressof(c), C.addressof(p), *a)

    assert f(None, C.addressof(good[1]), *ok) == f(C.addressof(good[0]), None, *ok) == B.ERR_INVALID_ARG
    for bad in (_cache(kv, size=8), _cache(kv, codes=None), _cache(kv, codes=FAKE + 8), _cache(kv, scale=None), _cache(kv, scale=FAKE + 4)):
        assert call(cache=bad) == B.ERR_INVALID_ARG
    for bad in (_cache(kv, n_pages=0), _cache(kv, heads=0), _cache(kv, dim=72), _cache(kv, page=40)):
        assert call(cache=bad) == B.ERR_SHAPE
    for bad in (_plan(kv, size=8), _plan(kv, tables=None), _plan(kv, held=None), _plan(kv, held=FAKE + 2), _plan(kv, index=None),
                _plan(kv, index=FAKE + 4)):
        assert call(plan=bad) == B.ERR_INVALID_ARG
    assert call(plan=_plan(kv, max_pages=0)) == B.ERR_SHAPE
    assert call(plan=_plan(kv, max_pages=2 ** 30)) == B.ERR_SHAPE           # positions past 2^30
    odd = _plan(kv)
    odd.small_rows = 17
    assert call(plan=odd) == B.ERR_SHAPE
    for i in (2, 5) if not attend else (2, 5, 9):                           # rows (q, out, workspace)
        i = {2: 1, 5: 4}[i] if not attend else i
        assert call(**{f"a{i}": None}) == call(**{f"a{i}": FAKE + 8}) == B.ERR_INVALID_ARG
    for i in (3, 4, 6, 7) if attend else (2, 3, 5, 6):                      # strides that leave rows misaligned
        assert call(**{f"a{i}": 132}) == B.ERR_SHAPE
    assert call(**{f"a{11 if attend else 7}": None}) == B.ERR_INVALID_ARG   # status
    if attend:
        for bad in (0.0, -1.0, float("nan"), 1e31):
            assert call(a0=bad) == B.ERR_INVALID_ARG
        assert call(a1=-1) == B.ERR_INVALID_ARG and call(a8=FAKE + 2) == B.ERR_INVALID_ARG
    else:
        assert call(a0=2) == B.ERR_INVALID_ARG
    assert call(plan=_plan(kv, lengths=(0, 0))) == B.OK                     # no rows: nothing to do


def test_numbers_of_a_plan_that_are_refused(kv):
    """Held positions and pages are whole numbers of 32 bits: nothing is wrapped around."""
    from paper_2605_11222_b200.binding import AdmmqError
    for good in ([], [[], []], [3, -1], np.array([5, 7], np.uint8), np.array([2 ** 31 - 1, -2 ** 31]), [[1, 2], [3, 4]], range(3)):
        a = kv._host(good, np.int32, "held")
        assert (a == np.asarray(good)).all() and a.dtype == np.int32
    for bad in (np.array([2 ** 32 + 5]), [np.int64(2 ** 32 + 5)], [2 ** 31], [-2 ** 31 - 1], [2 ** 70], [float("nan")], [float("inf")],
                [[1, 2], [3]], ["one"], [None], np.array([1.5])):
        with pytest.raises(AdmmqError):
            kv._host(bad, np.int32, "held")
    for bad in ([2 ** 70], [np.int64(2 ** 32 + 5)], np.array([2 ** 63 + 1], np.uint64), [[1, 2], [3]], ["one"], [None], [float("nan")]):
        with pytest.raises(AdmmqError):
            kv.CachePlan(bad, [0] * len(bad), [[0]] * len(bad))
    with pytest.raises(AdmmqError):
        kv.CachePlan([1], np.array([2 ** 32 + 5]), [[0]])
    with pytest.raises(AdmmqError):
        kv.CachePlan([1, 1], [0, 0], [[0, 1], [2]])


def test_outputs_whose_rows_or_heads_overlap_are_refused(kv):
    from paper_2605_11222_b200 import binding as B
    lib = kv._library()
    cache, plan = _cache(kv), _plan(kv)

    def read(k_row, k_head, v_row=128, v_head=64):
        return lib.admmq_cache_read(C.addressof(cache), C.addressof(plan), 1, None, k_row, k_head, FAKE, v_row, v_head, FAKE, None)

    def attend(row, head):
        return lib.admmq_cache_attend(C.addressof(cache), C.addressof(plan), 0.125, 0, None, 0, 0, FAKE, row, head, FAKE, FAKE, 0, FAKE, None)

    # six rows, two key heads, four query heads of 64; what fits is refused for its null pointer only
    for row, head in ((128, 64), (256, 64), (64, 384), (72, 432), (136, 72)):
        assert read(row, head) == B.ERR_INVALID_ARG
    for row, head in ((0, 64), (128, 0), (128, 72), (120, 64), (64, 64), (128, 56), (64, 376), (-128, 64)):
        assert read(row, head) == read(128, 64, row, head) == B.ERR_SHAPE
    for row, head in ((256, 64), (320, 72), (64, 384)):
        assert attend(row, head) == B.ERR_INVALID_ARG
    for row, head in ((0, 64), (256, 0), (248, 64), (256, 56), (64, 376)):
        assert attend(row, head) == B.ERR_SHAPE

"""GPU tests of the 8-bit cache of keys and values (kvcache.py) against its definition in cache_reference.py."""
import math

import pytest
import torch

from tests.cache_reference import ReferenceCache, attend64

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _rows(g, n, heads, d, dtype=torch.bfloat16):
    x = torch.randn(n, heads, d, generator=g, device=DEV)
    x[..., :: 37] *= 6.0
    return x.to(dtype)


def _tables(lengths, page, seed=0, spare=2):
    """Pages of every request, shuffled; (number of pages, lists, padded to one width with pages that do not exist)."""
    need = [-(-n // page) for n in lengths]
    order = torch.randperm(sum(need) + spare, generator=torch.Generator().manual_seed(seed)).tolist()
    lists = [order[sum(need[:i]): sum(need[: i + 1])] for i in range(len(need))]
    wide = max(1, max(need))
    return len(order), lists, [t + [2 ** 30] * (wide - len(t)) for t in lists]


class Setup:
    """A cache and its reference, filled up to `held` in one or several calls."""

    def __init__(self, lengths, held, heads, d, page, seed=1, steps=1, group=1, dtype=torch.bfloat16):
        from paper_2605_11222_b200 import kvcache
        g = self.g = _gen(seed)
        total = [n + max(0, p) for n, p in zip(lengths, held)]
        pages, self.lists, self.padded = _tables(total, page, seed)
        self.cache, self.ref = kvcache.KVCache(pages, heads, d, page, DEV), ReferenceCache(heads, d, page)
        self.cache.codes.random_(0, 256)                     # whatever was there before
        self.cache.scale.fill_(float("nan"))
        self.lengths, self.held, self.heads, self.d, self.group = lengths, held, heads, d, group
        done = [0] * len(held)
        for s in range(steps):
            n = [(max(0, p) * (s + 1)) // steps - a for p, a in zip(held, done)]
            if sum(n):
                self.write(n, done, _rows(g, sum(n), heads, d, dtype), _rows(g, sum(n), heads, d, dtype))
            done = [a + b for a, b in zip(done, n)]
        self.plan = kvcache.CachePlan(lengths, held, self.padded, group, DEV)

    def write(self, lengths, held, k, v):
        from paper_2605_11222_b200 import kvcache
        self.cache.write(k, v, kvcache.CachePlan(lengths, held, self.padded, device=DEV))
        self.ref.write(k, v, lengths, held, self.lists)

    def new_rows(self, dtype=torch.bfloat16):
        k, v = [_rows(self.g, sum(self.lengths), self.heads, self.d, dtype) for _ in "kv"]
        self.cache.write(k, v, self.plan)
        self.ref.write(k, v, self.lengths, self.held, self.lists)

    def sequences(self):
        return [tuple(self.ref.sequence(w, t, p + n) for w in "kv") if p >= 0 else None
                for t, p, n in zip(self.lists, self.held, self.lengths)]

    def check_attend(self, window=0, scale=None, q=None):
        from paper_2605_11222_b200 import adapt
        if q is None:
            q = (1.5 * torch.randn(sum(self.lengths), self.heads * self.group, self.d, generator=self.g, device=DEV)).bfloat16()
        out, lse = self.cache.attend(q, self.plan, scale, window)
        adapt.check_device_status(DEV)
        want = attend64(q, self.sequences(), self.lengths, self.held, self.group, scale or self.d ** -0.5, window)
        _within(out, want[0], want[2])
        _within(lse, want[1], want[3])
        return q, out, lse


def _within(got, want, tol):
    got = got.double().cpu()
    assert torch.equal(torch.isfinite(got), torch.isfinite(want))
    fine = torch.isfinite(want)
    assert torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)])
    err = (got - want).abs()[fine] / tol[fine].clamp(min=1e-300)
    worst = err.max().item() if err.numel() else 0.0
    assert worst <= 1.0, f"error is {worst:.3g} of the tolerance"


# (lengths, held, heads, head_dim, page, calls that fill the cache, type)
STORE = [
    ([1], [0], 1, 16, 16, 1, torch.bfloat16),
    ([1], [1003], 8, 128, 64, 1, torch.bfloat16),
    ([1, 1, 1, 1], [15, 16, 17, 0], 3, 64, 16, 9, torch.float32),
    ([5, 0, 40, 1], [3, 7, 30, 100], 2, 96, 32, 5, torch.bfloat16),
    ([33, 17], [0, 15], 5, 80, 128, 3, torch.float32),
    ([130], [61], 2, 256, 256, 7, torch.bfloat16),
    ([70], [2], 4, 192, 16, 1, torch.float32),
    ([3, 3], [-1, 20], 2, 112, 32, 20, torch.bfloat16),
]


@pytest.mark.parametrize("lengths,held,heads,d,page,steps,dtype", STORE)
def test_rows_are_kept_as_defined(lengths, held, heads, d, page, steps, dtype):
    """Codes and scales exactly: fp32 rows are read back as the definition's product, bf16 ones as its rounding."""
    from paper_2605_11222_b200 import adapt, kvcache
    s = Setup(lengths, held, heads, d, page, steps=steps, dtype=dtype)
    s.new_rows(dtype)
    begin = [max(0, p) for p in held]
    whole = [b + n if p >= 0 else 0 for b, n, p in zip(begin, lengths, held)]
    plan = kvcache.CachePlan(whole, [0] * len(whole), s.padded, device=DEV)
    k, v = s.cache.read(plan, torch.float32)
    kb, vb = s.cache.read(plan)
    adapt.check_device_status(DEV)
    for got, half, which in ((k, kb, "k"), (v, vb, "v")):
        want = s.ref.rows(which, whole, [0] * len(whole), s.lists)
        assert torch.equal(got.cpu(), want.float())
        assert torch.equal(half.cpu(), want.float().bfloat16())
    # the plan's own rows; those of a request that takes no part read as zero
    k, v = s.cache.read(s.plan, torch.float32)
    assert torch.equal(k.cpu(), s.ref.rows("k", lengths, held, s.lists).float())
    assert torch.equal(v.cpu(), s.ref.rows("v", lengths, held, s.lists).float())


# (lengths, held, heads, group, head_dim, page, window)
ATTEND = [
    ([1], [0], 1, 1, 16, 16, 0),
    ([1], [1], 2, 4, 64, 16, 0),
    ([1], [31], 1, 16, 128, 64, 0),
    ([1], [1000], 8, 4, 128, 64, 0),
    ([1, 1, 1], [5, 700, 31], 3, 5, 96, 32, 0),
    ([1, 1], [3000, -1], 2, 8, 128, 128, 500),
    ([1, 0, 1, 1], [40, 9, 41, 0], 2, 7, 80, 16, 33),
    ([1], [300], 1, 32, 64, 256, 0),
    ([3, 2, 4], [1000, 0, 77], 2, 4, 64, 16, 100),
    ([9], [2000], 2, 3, 128, 32, 0),
    ([5], [10], 2, 1, 256, 64, 0),
    ([1, 1], [513, 90], 2, 2, 192, 64, 0),
    ([1, 1], [513, 90], 2, 2, 240, 64, 64),
    ([33, 1, 70], [0, 200, 100], 2, 3, 128, 64, 0),
    ([128], [0], 1, 2, 128, 64, 0),
    ([300, 1, 257], [100, 400, 0], 2, 4, 64, 32, 0),
    ([130, 260], [3, 1000], 1, 5, 96, 128, 200),
    ([200], [64], 2, 2, 256, 64, 0),
    ([150], [500], 1, 3, 192, 16, 70),
    ([600], [0], 1, 1, 128, 64, 1),
    ([40, 90], [-1, 700], 2, 8, 112, 64, 0),
]


@pytest.mark.parametrize("lengths,held,heads,group,d,page,window", ATTEND)
def test_attention_matches_the_formula(lengths, held, heads, group, d, page, window):
    s = Setup(lengths, held, heads, d, page, seed=sum(held) + d, group=group)
    s.new_rows()
    s.check_attend(window)


@pytest.mark.parametrize("lengths,held,heads,group,d,window", [
    ([1] * 70, [(37 * i) % 900 for i in range(70)], 8, 4, 128, 0),          # more (tile, head)s than CTAs
    ([1] * 30, [(211 * i) % 2500 for i in range(30)], 3, 2, 64, 700),       # fewer
    ([2, 1, 5, 1] * 5, [(97 * i) % 1500 for i in range(20)], 4, 3, 96, 0),
    ([70 + 13 * (i % 9) for i in range(24)], [(131 * i) % 700 for i in range(24)], 8, 1, 64, 0),
    ([100, 1, 90, 1, 1], [30, 1200, 500, 77, 3000], 2, 4, 128, 256),
    ([64] * 9, [300 * i for i in range(9)], 2, 4, 256, 0),
])
def test_work_shared_out_over_ragged_requests(lengths, held, heads, group, d, window):
    s = Setup(lengths, held, heads, d, 32, seed=len(lengths), group=group)
    s.new_rows()
    q, out, lse = s.check_attend(window)
    again = s.cache.attend(q, s.plan, window=window)                        # one order of every sum
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])


@pytest.mark.parametrize("lengths,held,heads,group,d,page,window", ATTEND + [
    ([1] * 20, [(137 * i) % 1100 for i in range(20)], 4, 4, 128, 64, 0),
    ([2] * 6, [400 * i for i in range(6)], 2, 8, 192, 32, 333)])
def test_tables_far_longer_than_the_requests(lengths, held, heads, group, d, page, window):
    from paper_2605_11222_b200 import kvcache
    s = Setup(lengths, held, heads, d, page, seed=sum(held) + d, group=group)
    s.new_rows()
    q, out, lse = s.check_attend(window)
    wide = [t + [2 ** 30] * (40000 // page) for t in s.padded]              # the call that may not count on short requests
    s.plan = kvcache.CachePlan(lengths, held, wide, group, DEV)
    s.check_attend(window, q=q)


@pytest.mark.parametrize("n,heads,d", [(1, 1, 128), (2, 8, 128), (5, 8, 64), (3, 9, 128), (9, 8, 128), (13, 8, 64), (27, 8, 128),
                                       (50, 8, 128), (50, 8, 64), (7, 8, 192), (14, 8, 256), (25, 8, 256)])
def test_numbers_of_requests(n, heads, d):
    held = [(29 * i + 61) % 400 for i in range(n - 1)] + [970]              # a long one: CTAs together from 16 down to one
    s = Setup([1] * n, held, heads, d, 64, seed=n, group=2)
    s.new_rows()
    s.check_attend()


def test_one_long_request_is_split_and_joined():
    s = Setup([1], [20000], 2, 128, 128, group=8, seed=3)                   # (over the clusters' positions)
    s.new_rows()
    s.check_attend()
    s.check_attend(window=19000)


@pytest.mark.parametrize("lengths,d", [([1, 3], 128), ([1, 3], 256), ([150, 70], 128), ([150, 70], 64), ([90, 40], 192)])
@pytest.mark.parametrize("kind", ["growing", "peaked", "value scales"])
def test_references_are_raised_and_scales_differ(lengths, d, kind):
    """Scores that go on growing raise a row's reference again and again, also within a step; one key takes nearly all of the
    weight; values of neighbouring blocks lie a million apart."""
    held = [700, 333]
    s = Setup(lengths, [0, 0], 2, d, 64, group=2, seed=d)
    total = [n + p for n, p in zip(lengths, held)]
    from paper_2605_11222_b200 import kvcache
    pages, s.lists, s.padded = _tables(total, 64, 5)
    s.cache = kvcache.KVCache(pages, 2, d, 64, DEV)
    s.ref = ReferenceCache(2, d, 64)
    k, v = [_rows(s.g, sum(total), 2, d).float() for _ in "kv"]
    at = torch.cat([torch.arange(n, device=DEV) for n in total])[:, None, None]
    direction = torch.randn(2, d, generator=s.g, device=DEV)
    if kind == "growing":
        k = 0.1 * k + direction * (at / 40.0) * (1 + (at % 29 == 0))
    elif kind == "peaked":
        k = torch.where(at == 200, 20.0 * direction, 0.3 * k)
    else:
        v = v * 10.0 ** (((at // 16) % 4) * 2 - 3)
    s.write(total, [0, 0], k.bfloat16(), v.bfloat16())
    s.held = held
    s.plan = kvcache.CachePlan(lengths, held, s.padded, 2, DEV)
    q = (0.3 * torch.randn(sum(lengths), 2, 2, d, generator=s.g, device=DEV) + direction[:, None]).reshape(-1, 4, d).bfloat16()
    s.check_attend(q=q)


@pytest.mark.parametrize("lengths", [[40], [1, 3], [130]])
def test_a_block_with_nan_reaches_only_rows_that_see_it(lengths):
    from paper_2605_11222_b200 import adapt
    held = [50] * len(lengths)
    s = Setup(lengths, held, 1, 64, 16, group=2)
    k, v = [_rows(s.g, sum(lengths), 1, 64) for _ in "kv"]
    v[0, 0, 5] = float("nan")                    # position 50 of the first request: block 3, tokens 48 .. 63
    s.cache.write(k, v, s.plan)
    s.ref.write(k, v, lengths, held, s.lists)
    q = torch.randn(sum(lengths), 2, 64, generator=s.g, device=DEV).bfloat16()
    out, lse = s.cache.attend(q, s.plan)
    bad = torch.zeros(sum(lengths), dtype=torch.bool, device=DEV)
    bad[: lengths[0]] = True                     # every new row sees token 48 or 50 of it
    assert torch.equal(torch.isnan(out).all(-1).all(-1), bad) and torch.equal(torch.isnan(out).any(-1).any(-1), bad)
    # a window that leaves the block out: rows from position 64 + 10 on
    out, lse = s.cache.attend(q, s.plan, window=11)
    pos = torch.cat([torch.arange(p, p + n) for n, p in zip(lengths, held)]).to(DEV)
    bad &= pos - 10 < 64
    assert torch.equal(torch.isnan(out).any(-1).any(-1), bad) and torch.isfinite(lse[~bad]).all()
    # rows before it, asked again
    from paper_2605_11222_b200 import kvcache
    early = kvcache.CachePlan([48], [0], s.padded[:1], 2, DEV)
    out, lse = s.cache.attend(torch.randn(48, 2, 64, generator=s.g, device=DEV).bfloat16(), early)
    assert torch.isfinite(out.float()).all() and torch.isfinite(lse).all()
    # the block starts anew
    fresh = kvcache.CachePlan([20], [48], s.padded[:1], device=DEV)
    if lengths[0] >= 18:
        s.cache.write(_rows(s.g, 20, 1, 64), _rows(s.g, 20, 1, 64), fresh)
        assert torch.isfinite(s.cache.attend(q[:1], kvcache.CachePlan([1], [60], s.padded[:1], 2, DEV))[0].float()).all()
    adapt.check_device_status(DEV)


@pytest.mark.parametrize("n", [1, 40])
def test_a_query_with_nan_or_infinity_stays_in_its_row(n):
    s = Setup([n, n], [100, 30], 2, 128, 64, group=2)
    s.new_rows()
    q = torch.randn(2 * n, 4, 128, generator=s.g, device=DEV).bfloat16()
    good = s.cache.attend(q, s.plan)
    q2 = q.clone()
    q2[0, 1, 7], q2[n, 2, 0] = float("inf"), float("nan")
    out, lse = s.cache.attend(q2, s.plan)
    for r, h in ((0, 1), (n, 2)):
        assert torch.isnan(out[r, h]).all() and torch.isnan(lse[r, h])
        out[r, h], lse[r, h] = good[0][r, h], good[1][r, h]
    assert torch.equal(out, good[0]) and torch.equal(lse, good[1])


def test_magnitudes_at_the_ends_of_the_range():
    """Below 2^-40 a block is held as zeros; from 2^40 on, or with an infinity or a NaN, it is NaN until it starts anew."""
    from paper_2605_11222_b200 import kvcache
    s = Setup([16] * 6, [0] * 6, 2, 32, 16)
    k, v = [_rows(s.g, 96, 2, 32, torch.float32) for _ in "kv"]
    k = k.clamp(-1, 1)
    k[0:16] *= 2.0 ** -41
    k[16:32] = (k[16:32] * 0.5) * 2.0 ** 40
    k[32, 1, 3] = 2.0 ** 40
    k[48, 0, 0] = float("inf")
    k[64, 1, 31] = float("nan")
    k[80:96] = 0.0
    s.cache.write(k, v, s.plan)
    s.ref.write(k, v, s.lengths, s.held, s.lists)
    got = s.cache.read(s.plan, torch.float32)[0].cpu()
    want = s.ref.rows("k", s.lengths, s.held, s.lists).float()
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got.nan_to_num(), want.nan_to_num())
    assert (got[0:16] == 0).all() and torch.isfinite(got[16:32]).all() and torch.isnan(got[32:48, 1]).all()
    assert torch.isfinite(got[32:48, 0]).all() and torch.isnan(got[48:64, 0]).all() and torch.isnan(got[64:80, 1]).all()
    one = kvcache.CachePlan([1] * 6, [0] * 6, s.padded, device=DEV)
    s.cache.write(torch.ones(6, 2, 32, device=DEV), torch.ones(6, 2, 32, device=DEV), one)
    assert (s.cache.read(one, torch.float32)[0] == 1).all()


def test_a_block_of_nan_stays_so_when_tokens_are_added():
    from paper_2605_11222_b200 import kvcache
    s = Setup([1], [3], 1, 64, 16)
    x = torch.full((1, 1, 64), float("nan"), device=DEV)
    s.cache.write(x, torch.ones_like(x), s.plan)
    after = kvcache.CachePlan([2], [4], s.padded, device=DEV)
    s.cache.write(torch.ones(2, 1, 64, device=DEV), torch.ones(2, 1, 64, device=DEV), after)
    k, v = s.cache.read(kvcache.CachePlan([6], [0], s.padded, device=DEV), torch.float32)
    assert torch.isnan(k).all() and torch.isfinite(v).all()


def test_strides_of_every_argument():
    from paper_2605_11222_b200 import adapt
    lengths, held = [5, 1, 60], [10, 200, 0]
    s = Setup(lengths, held, 3, 64, 32, group=2)
    t = sum(lengths)
    g = s.g
    wide = torch.randn(t, 2, 3 + 3 + 6, 80, generator=g, device=DEV).bfloat16()
    k, v, q = wide[:, 0, :3, :64], wide[:, 0, 3:6, :64], wide[:, 1, 6:, 8:72]
    s.cache.write(k, v, s.plan)
    s.ref.write(k, v, lengths, held, s.lists)
    out_buf, kv_buf = torch.full((t, 7, 96), 7.0, device=DEV).bfloat16(), torch.full((t, 8, 72), 7.0, device=DEV)
    out, lse = out_buf[:, :6, :64], torch.full((t, 6), 7.0, device=DEV)
    r = s.cache.attend(q, s.plan, out=out, lse=lse)
    assert r[0] is out and r[1] is lse
    want = s.cache.attend(q.contiguous(), s.plan)
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
    assert (out_buf[:, 6] == 7).all() and (out_buf[:, :, 64:] == 7).all()
    rk, rv = s.cache.read(s.plan, torch.float32, kv_buf[:, :3, 8:72], kv_buf[:, 4:7, 8:72])
    wk, wv = s.cache.read(s.plan, torch.float32)
    assert torch.equal(rk, wk) and torch.equal(rv, wv)
    assert torch.equal(wk.cpu(), s.ref.rows("k", lengths, held, s.lists).float())
    assert (kv_buf[:, 3] == 7).all() and (kv_buf[..., :8] == 7).all()
    # head-major keys
    k2 = torch.randn(3, t, 64, generator=g, device=DEV).transpose(0, 1)
    s.cache.write(k2, k2, s.plan)
    a = s.cache.read(s.plan, torch.float32)[0]
    s.cache.write(k2.contiguous(), k2.contiguous(), s.plan)
    assert torch.equal(a, s.cache.read(s.plan, torch.float32)[0])
    adapt.check_device_status(DEV)


@pytest.mark.parametrize("n", [1, 30, 100])
def test_requests_that_take_no_part_and_tables_that_do_not_hold(n):
    """held < 0, a table that is too short, a page that does not exist: the others' rows are as they would be alone."""
    from paper_2605_11222_b200 import adapt, kvcache
    from paper_2605_11222_b200.binding import AdmmqError
    lengths, held = [n, n, n], [40, 70, 33]
    s = Setup(lengths, held, 2, 64, 16, group=2)
    s.new_rows()
    q = torch.randn(3 * n, 4, 64, generator=s.g, device=DEV).bfloat16()
    want = s.cache.attend(q, s.plan)
    before = s.cache.read(s.plan)
    k = _rows(s.g, 3 * n, 2, 64)
    adapt.check_device_status(DEV)

    out_k = kvcache.CachePlan(lengths, [40, -1, 33], s.padded, 2, DEV)
    out, lse = s.cache.attend(q, out_k)
    assert (out[n: 2 * n] == 0).all() and (lse[n: 2 * n] == -math.inf).all()
    for got, w in ((out, want[0]), (lse, want[1])):
        assert torch.equal(got[:n], w[:n]) and torch.equal(got[2 * n:], w[2 * n:])
    got = s.cache.read(out_k)[0]
    assert (got[n: 2 * n] == 0).all() and torch.equal(got[:n], before[0][:n])
    adapt.check_device_status(DEV)

    long_held = [40, 16 * len(s.padded[0]) - n + 1, 33]
    bad_table = [list(r) for r in s.padded]
    bad_table[1][2] = 10 ** 6
    neg_table = [list(r) for r in s.padded]
    neg_table[1][3] = -1
    for plan in (kvcache.CachePlan(lengths, long_held, s.padded, 2, DEV), kvcache.CachePlan(lengths, held, bad_table, 2, DEV),
                 kvcache.CachePlan(lengths, held, neg_table, 2, DEV)):
        out, lse = s.cache.attend(q, plan)
        assert torch.equal(out[:n], want[0][:n]) and torch.equal(out[2 * n:], want[0][2 * n:])
        with pytest.raises(AdmmqError):
            adapt.check_device_status(DEV)
    plan = kvcache.CachePlan(lengths, long_held, s.padded, 2, DEV)
    s.cache.write(k, k, plan)                                                # nothing of request 1
    with pytest.raises(AdmmqError):
        adapt.check_device_status(DEV)
    assert torch.equal(s.cache.read(s.plan)[0][n: 2 * n], before[0][n: 2 * n])
    adapt.check_device_status(DEV)


def test_pages_that_two_requests_read():
    """A shared prefix: two requests' tables name the same pages for it."""
    s = Setup([1], [200], 2, 64, 32, group=4)
    s.new_rows()
    from paper_2605_11222_b200 import kvcache
    q = torch.randn(2, 8, 64, generator=s.g, device=DEV).bfloat16()
    both = kvcache.CachePlan([1, 1], [200, 150], s.padded + s.padded, 4, DEV)
    out, lse = s.cache.attend(q, both)
    a = s.cache.attend(q[:1], kvcache.CachePlan([1], [200], s.padded, 4, DEV))
    b = s.cache.attend(q[1:], kvcache.CachePlan([1], [150], s.padded, 4, DEV))
    for got, x, y in ((out, a[0], b[0]), (lse, a[1], b[1])):
        assert (got[:1] - x).abs().max() <= 2.0 ** -7 * x.abs().max() and (got[1:] - y).abs().max() <= 2.0 ** -7 * y.abs().max()


def test_no_rows():
    from paper_2605_11222_b200 import kvcache
    cache = kvcache.KVCache(4, 2, 64, 16, DEV)
    plan = kvcache.CachePlan([0, 0], [3, 5], [[0, 1], [2, 3]], 3, DEV)
    e = torch.empty(0, 2, 64, dtype=torch.bfloat16, device=DEV)
    cache.write(e, e, plan)
    assert cache.read(plan)[0].shape == (0, 2, 64)
    out, lse = cache.attend(torch.empty(0, 6, 64, dtype=torch.bfloat16, device=DEV), plan)
    assert out.shape == (0, 6, 64) and lse.shape == (0, 6)


def test_a_captured_step_follows_the_device():
    """One graph of a decoding step, replayed: the positions move on, a request drops out, on a stream of its own."""
    from paper_2605_11222_b200 import adapt, kvcache
    steps, page = 20, 16
    s = Setup([1, 1, 1], [30, 0, 77], 2, 64, page, group=2)
    total = [30 + steps, steps, 77 + steps]
    pages, lists, padded = _tables(total, page, 9)
    cache, ref = kvcache.KVCache(pages, 2, 64, page, DEV), ReferenceCache(2, 64, page)
    fill = _rows(s.g, 107, 2, 64)
    cache.write(fill, fill, kvcache.CachePlan([30, 0, 77], [0, 0, 0], padded, device=DEV))
    ref.write(fill, fill, [30, 0, 77], [0, 0, 0], lists)
    plan = kvcache.CachePlan([1, 1, 1], torch.tensor([30, 0, 77], dtype=torch.int32, device=DEV),
                             torch.tensor(padded, dtype=torch.int32, device=DEV), 2)
    k, v, q = [torch.zeros(3, h, 64, dtype=torch.bfloat16, device=DEV) for h in (2, 2, 4)]
    out, lse = torch.zeros(3, 4, 64, dtype=torch.bfloat16, device=DEV), torch.zeros(3, 4, device=DEV)

    def step():
        cache.write(k, v, plan)
        cache.attend(q, plan, out=out, lse=lse)
        plan.held += 1

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    held = [30, 0, 77]
    with torch.cuda.stream(stream):
        step()                                               # (a first call, with rows of zeros)
        stream.synchronize()
        plan.held -= 1
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            step()
        for i in range(steps):
            nk, nv, nq = [torch.randn(3, h, 64, generator=s.g, device=DEV).bfloat16() for h in (2, 2, 4)]
            if i == 12:
                plan.held[1] = -100
                held[1] = -1
            torch.cuda.synchronize()
            k.copy_(nk), v.copy_(nv), q.copy_(nq)
            graph.replay()
            stream.synchronize()
            ref.write(nk, nv, [1, 1, 1], held, lists)
            seqs = [tuple(ref.sequence(w, t, p + 1) for w in "kv") if p >= 0 else None for t, p in zip(lists, held)]
            want = attend64(nq, seqs, [1, 1, 1], held, 2, 0.125)
            _within(out, want[0], want[2])
            _within(lse, want[1], want[3])
            held = [p + 1 if p >= 0 else p for p in held]
    adapt.check_device_status(DEV)


def test_two_streams_at_once():
    a, b = [Setup([1, 100], [500, 0], 4, 128, 64, group=2, seed=i) for i in (1, 2)]
    for s in (a, b):
        s.new_rows()
    qs = [torch.randn(101, 8, 128, generator=s.g, device=DEV).bfloat16() for s in (a, b)]
    want = [s.cache.attend(q, s.plan) for s, q in zip((a, b), qs)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in "ab"]
    got = [[], []]
    for _ in range(20):
        for i, s in enumerate((a, b)):
            with torch.cuda.stream(streams[i]):
                got[i].append(s.cache.attend(qs[i], s.plan))
    torch.cuda.synchronize()
    for w, g in zip(want, got):
        assert all(torch.equal(w[0], o) and torch.equal(w[1], l) for o, l in g)


@pytest.mark.parametrize("lengths,held", [([1], [100]), ([1] * 40, [100] * 40), ([200], [100])])
def test_waits_run_out(lengths, held):
    """With no codes on their way every wait ends at its limit, the call says so, and the next one works."""
    from paper_2605_11222_b200 import adapt
    from paper_2605_11222_b200.binding import AdmmqError, ERR_TIMEOUT
    s = Setup(lengths, held, 8, 128, 64, group=2)
    s.new_rows()
    q = torch.randn(sum(lengths), 16, 128, generator=s.g, device=DEV).bfloat16()
    want = s.cache.attend(q, s.plan)
    lib = adapt._library()
    assert lib.admmq_test_linear_set_wait(2_000_000, 1) == 0
    try:
        s.cache.attend(q, s.plan)
        with pytest.raises(AdmmqError) as e:
            adapt.check_device_status(DEV)
        assert e.value.status == ERR_TIMEOUT
    finally:
        assert lib.admmq_test_linear_set_wait(2_000_000_000, 0) == 0
    out, lse = s.cache.attend(q, s.plan)
    adapt.check_device_status(DEV)
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


def test_calls_refuse_bad_arguments():
    from paper_2605_11222_b200 import kvcache
    from paper_2605_11222_b200.binding import AdmmqError
    for bad in ((0, 2, 64, 16), (4, 0, 64, 16), (4, 2, 72, 16), (4, 2, 272, 16), (4, 2, 64, 24), (4, 2, 64, 512), (4, 5000, 64, 16)):
        with pytest.raises(AdmmqError):
            kvcache.KVCache(*bad, DEV)
    table = [[0, 1], [2, 3]]
    for bad in (([], [], table), ([1, -1], [0, 0], table), ([1, 1], [0], table), ([1, 1], [0, 0], table[:1]), ([1, 1], [0, 0], [[], []])):
        with pytest.raises(AdmmqError):
            kvcache.CachePlan(*bad, device=DEV)
    for group in (0, -1, 2000):
        with pytest.raises(AdmmqError):
            kvcache.CachePlan([1, 1], [0, 0], table, group, DEV)
    with pytest.raises(AdmmqError):
        kvcache.CachePlan([1, 1], torch.zeros(2, dtype=torch.int64, device=DEV), table, device=DEV)
    cache, plan = kvcache.KVCache(4, 2, 64, 16, DEV), kvcache.CachePlan([1, 1], [0, 0], table, 2, DEV)
    k = torch.zeros(2, 2, 64, dtype=torch.bfloat16, device=DEV)
    q = torch.zeros(2, 4, 64, dtype=torch.bfloat16, device=DEV)
    odd = torch.zeros(2, 2, 68, dtype=torch.bfloat16, device=DEV)[..., 4:]                       # 8 bytes off
    for bad in (k[:1], k[:, :1], k[..., :32], k.half(), k.cpu(), k.transpose(1, 2), k.view(4, 64), odd,
                torch.zeros(2, 64, 2, dtype=torch.bfloat16, device=DEV).transpose(1, 2)):
        with pytest.raises(AdmmqError):
            cache.write(bad, k, plan)
        with pytest.raises(AdmmqError):
            cache.write(k, bad, plan)
        with pytest.raises(AdmmqError):
            cache.read(plan, k=bad)
    with pytest.raises(AdmmqError):
        cache.write(k, k.float(), plan)
    for bad in (q[:1], q[:, :3], q.float(), q.cpu(), k):
        with pytest.raises(AdmmqError):
            cache.attend(bad, plan)
        with pytest.raises(AdmmqError):
            cache.attend(q, plan, out=bad)
    for kw in (dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(window=-1), dict(window=2 ** 40), dict(lse=torch.zeros(2, 3, device=DEV)),
               dict(lse=torch.zeros(2, 4, device=DEV, dtype=torch.float64))):
        with pytest.raises(AdmmqError):
            cache.attend(q, plan, **kw)
    with pytest.raises(AdmmqError):
        cache.read(plan, torch.float16)
    for call in (lambda p: cache.write(k, k, p), lambda p: cache.read(p), lambda p: cache.attend(q, p)):
        with pytest.raises(AdmmqError):
            call(None)
    for x in (k, q):
        y = x.clone().requires_grad_()
        with pytest.raises(AdmmqError):
            cache.write(y, k, plan) if x is k else cache.attend(y, plan)
        with torch.no_grad():
            cache.write(y, k, plan) if x is k else cache.attend(y, plan)
    # other storage than when they were made
    held = plan.held.clone()
    plan.held.data = held
    with pytest.raises(AdmmqError):
        cache.attend(q, plan)
    plan2 = kvcache.CachePlan([1, 1], [0, 0], table, 2, DEV)
    cache.scale.data = cache.scale.clone()
    with pytest.raises(AdmmqError):
        cache.write(k, k, plan2)


def test_given_scale_and_unrolled_decoding_agree_with_a_prompt():
    """The rows of a prompt, one at a time behind each other, are within the tolerances of the formula on what the cache
    holds at the time; the prompt's rows on what it holds in the end."""
    n = 40
    s = Setup([n], [0], 2, 96, 32, group=2)
    s.new_rows()
    s.check_attend(scale=0.2)
    one = Setup([1], [0], 2, 96, 32, group=2)
    from paper_2605_11222_b200 import kvcache
    pages, one.lists, one.padded = _tables([n], 32, 1)
    one.cache, one.ref = kvcache.KVCache(pages, 2, 96, 32, DEV), ReferenceCache(2, 96, 32)
    for i in range(n):
        one.held, one.plan = [i], kvcache.CachePlan([1], [i], one.padded, 2, DEV)
        one.new_rows()
        one.check_attend(window=17)


def test_a_block_runs_its_prompts_and_decodes():
    """Projections from codes with adapters, norm and rotation, cache and attention together, as a served block calls them:
    prompts of ragged requests, then tokens one by one, one request joined by another in between."""
    from paper_2605_11222_b200 import adapt, kvcache
    heads, kv, d, hidden, page = 8, 2, 64, 512, 16
    g = _gen(5)
    layers, banks = [], []
    for p in (heads * d, kv * d, kv * d):
        codes = torch.randint(0, 16, (p, hidden), generator=g, device=DEV).to(torch.uint8)
        scale = torch.full((p, 4), 0.06 / 15, device=DEV) * (1 + torch.rand(p, 4, generator=g, device=DEV))
        layers.append(adapt.QuantLinear(codes, scale, -7.5 * scale, 4, 128))
        banks.append(adapt.AdapterBank((0.05 * torch.randn(2, 8, hidden, generator=g, device=DEV)).bfloat16(),
                                       (0.05 * torch.randn(2, 8, p, generator=g, device=DEV)).bfloat16(), torch.ones(2, device=DEV)))
    w = [(1 + 0.1 * torch.randn(d, generator=g, device=DEV)).bfloat16() for _ in "qk"]
    ang = torch.arange(256, device=DEV)[:, None] * 1e4 ** (-torch.arange(0, d, 2, device=DEV) / d)
    cos, sin = ang.cos(), ang.sin()
    lengths, adapters = [70, 0, 3, 33], [0, -1, 1, -1]
    total = [n + 6 for n in lengths]
    pages, lists, padded = _tables(total, page, 3)
    cache, ref = kvcache.KVCache(pages, kv, d, page, DEV), ReferenceCache(kv, d, page)
    tables = torch.tensor(padded, dtype=torch.int32, device=DEV)
    held = [0, 0, 0, 0]

    def run(new):
        requests = adapt.RequestPlan(new, adapters, 2, DEV)
        x = torch.randn(requests.n_rows, hidden, generator=g, device=DEV).bfloat16()
        q, k, v = [l.forward(x, b, requests)[0] for l, b in zip(layers, banks)]
        pos = torch.cat([torch.arange(p, p + n, dtype=torch.int32) for p, n in zip(held, new)]).to(DEV)
        q, k = adapt.qk_norm_rope(q.view(-1, heads, d), k.view(-1, kv, d), *w, cos, sin, pos)
        plan = kvcache.CachePlan(new, held, tables, heads // kv)
        v = v.view(-1, kv, d)
        cache.write(k, v, plan)
        out, lse = cache.attend(q, plan)
        adapt.check_device_status(DEV)
        ref.write(k, v, new, held, lists)
        seqs = [tuple(ref.sequence(s, t, p + n) for s in "kv") for t, p, n in zip(lists, held, new)]
        want = attend64(q, seqs, new, held, heads // kv, d ** -0.5)
        _within(out, want[0], want[2])
        _within(lse, want[1], want[3])
        return [p + n for p, n in zip(held, new)]

    held = run(lengths)
    held = run([1, 0, 1, 1])
    held = run([1, 5, 1, 1])                     # the empty request's prompt joins the decoding ones
    for _ in range(3):
        held = run([1, 1, 1, 1])

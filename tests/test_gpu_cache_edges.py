"""GPU tests of the 8-bit cache where attention over it meets the ends of its ranges: pieces of calls whose waits run out,
blocks of zeros, weights far below a row's largest, pages behind a window, queries near zero."""
import ctypes as C
import math

import pytest
import torch

from tests.cache_reference import ReferenceCache, attend64
from tests.test_gpu_cache import DEV, Setup, _gen, _rows, _tables, _within

pytestmark = pytest.mark.gpu


def test_waits_that_run_out_leave_nothing_to_be_joined_untold():
    """A call whose joins go by (tile, head), some CTAs with more of them than wait to be taken at once: when the waits
    run out, all of them have been told to the join, which uses what it finds as indexes.  The workspace holds harmless entries
    (nothing to be joined) with a mark where a told one has zeros."""
    from paper_2605_11222_b200 import adapt, kvcache
    from paper_2605_11222_b200.binding import ERR_TIMEOUT, AdmmqError
    heads, group, d, page, short, at = 8, 4, 64, 64, 17, 60000
    lengths, held = [40] * (short + 1), [at] + [0] * short
    wide = -(-(at + 40) // page)
    tables = [list(range(wide))] + [[wide + i] + [0] * (wide - 1) for i in range(short)]
    cache = kvcache.KVCache(wide + short, heads, d, page, DEV)
    cache.codes.random_(1, 256, generator=_gen(1))
    cache.scale.fill_(0.01)
    plan = kvcache.CachePlan(lengths, held, tables, group, DEV)
    pieces = (short + 1) * heads                     # 160 packed rows: one tile of many rows a request
    assert plan._c.n_small == 0 and plan._c.n_big == short + 1
    ctas = torch.cuda.get_device_properties(DEV).multi_processor_count
    assert pieces <= ctas
    q = torch.randn(plan.n_rows, heads * group, d, generator=_gen(2), device=DEV).bfloat16()
    want = cache.attend(q, plan)
    adapt.check_device_status(DEV)

    lib = kvcache._library()
    nbytes = lib.admmq_cache_attend_workspace(cache._ref, plan._ref)
    work = torch.zeros(nbytes // 4, dtype=torch.int32, device=DEV)
    entries = work[: 8 * pieces].view(pieces, 8)     # first, last, head, row0, first row, rows, two of padding
    entries[:, 6:] = 77
    out, lse = torch.zeros_like(q), torch.zeros(plan.n_rows, heads * group, device=DEV)

    def call():
        adapt._call(lib.admmq_cache_attend, "admmq_cache_attend", 0, cache._ref, plan._ref, d ** -0.5, 0, q.data_ptr(), heads * group * d,
                    d, out.data_ptr(), heads * group * d, d, lse.data_ptr(), work.data_ptr(), C.c_size_t(nbytes), cache._status)

    assert lib.admmq_test_linear_set_wait(2_000_000, 1) == 0
    try:
        call()
        with pytest.raises(AdmmqError) as e:
            adapt.check_device_status(DEV)
        assert e.value.status == ERR_TIMEOUT
    finally:
        assert lib.admmq_test_linear_set_wait(2_000_000_000, 0) == 0
    told = entries.cpu()
    assert (told[:, 6:] == 0).all()
    assert (told[:, 0] >= 0).all() and (told[:, 1] >= told[:, 0]).all() and (told[:, 1] < ctas).all()
    assert told[:, 2].tolist() == [i % heads for i in range(pieces)] and (told[:, 3] == 0).all()
    assert told[:, 4].tolist() == [40 * (i // heads) for i in range(pieces)] and (told[:, 5] == 160).all()
    call()                                           # and the same workspace serves the next call
    adapt.check_device_status(DEV)
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


@pytest.mark.parametrize("d", [64, 128, 192])
def test_references_that_rise_at_every_step_give_the_same_bits(d):
    """Scores that go on growing make the two threads of a row agree on a new reference again and again: fifty calls of three
    requests at once, one result."""
    from paper_2605_11222_b200 import adapt, kvcache
    lengths, held, page = [150, 70, 200], [3000, 1000, 0], 64
    total = [n + p for n, p in zip(lengths, held)]
    need = [-(-n // page) for n in total]
    tables = [[sum(need[:i]) + j if j < need[i] else 0 for j in range(max(need))] for i in range(3)]
    cache, g = kvcache.KVCache(sum(need), 4, d, page, DEV), _gen(d)
    direction = torch.randn(4, d, generator=g, device=DEV)
    at = torch.cat([torch.arange(n, device=DEV) for n in total])[:, None, None]
    k = 0.1 * torch.randn(sum(total), 4, d, generator=g, device=DEV) + direction * (at / 40.0)
    cache.write(k.bfloat16(), torch.randn(sum(total), 4, d, generator=g, device=DEV).bfloat16(),
                kvcache.CachePlan(total, [0] * 3, tables, device=DEV))
    plan = kvcache.CachePlan(lengths, held, tables, 2, DEV)
    q = direction.repeat_interleave(2, 0) + 0.3 * torch.randn(plan.n_rows, 8, d, generator=g, device=DEV)
    q = q.bfloat16()
    want = cache.attend(q, plan)
    got = [cache.attend(q, plan) for _ in range(50)]
    adapt.check_device_status(DEV)
    assert torch.isfinite(want[0].float()).all()
    assert all(torch.equal(o, want[0]) and torch.equal(l, want[1]) for o, l in got)


# packed rows of few and of many, heads of one track and of two, requests in clusters and shared out
FORMS = [([1], 128, 300), ([1, 3], 256, 300), ([2] * 40, 64, 200), ([130], 64, 300), ([150, 70], 128, 200), ([90, 40], 192, 300)]


@pytest.mark.parametrize("lengths,d,held", FORMS)
@pytest.mark.parametrize("size", [1e-3, 1e-5, 1e-9])
@pytest.mark.parametrize("zeros", [(0, 16), (32, 48), (160, 176), (0, 64), (200, 201)])
def test_a_block_of_zero_values_leaves_its_neighbours_their_digits(lengths, d, held, size, zeros):
    """Values of one size, and a block of them zero or below 2^-40 (its scale is 0): it has weight in the sum and none in the
    result, and what scale the kernels take it to have must not push the others' weights out of their 16 bits."""
    s = Setup(lengths, [0] * len(lengths), 2, d, 64, seed=d, group=2)
    total = [n + held for n in lengths]
    from paper_2605_11222_b200 import kvcache
    pages, s.lists, s.padded = _tables(total, 64, 5)
    s.cache, s.ref = kvcache.KVCache(pages, 2, d, 64, DEV), ReferenceCache(2, d, 64)
    k, v = [_rows(s.g, sum(total), 2, d).float() for _ in "kv"]
    at = torch.cat([torch.arange(n, device=DEV) for n in total])[:, None, None]
    gone = (at >= zeros[0]) & (at < zeros[1])
    v = torch.where(gone, 1e-14 * v if zeros[0] == 32 else 0.0 * v, size * v)
    s.write(total, [0] * len(lengths), k.bfloat16(), v.bfloat16())
    s.held = [held] * len(lengths)
    s.plan = kvcache.CachePlan(lengths, s.held, s.padded, 2, DEV)
    q = (0.3 * torch.randn(sum(lengths), 4, d, generator=s.g, device=DEV)).bfloat16()
    out, lse = s.cache.attend(q, s.plan)
    want = attend64(q, s.sequences(), lengths, s.held, 2, d ** -0.5)
    _within(out, want[0], want[2])
    _within(lse, want[1], want[3])


@pytest.mark.parametrize("lengths,d", [([1], 128), ([1, 3], 256), ([130], 64), ([90], 192)])
def test_values_that_are_all_zero(lengths, d):
    s = Setup(lengths, [100] * len(lengths), 2, d, 64, group=2)
    total = [n + 100 for n in lengths]
    k, v = _rows(s.g, sum(total), 2, d), torch.zeros(sum(total), 2, d, device=DEV).bfloat16()
    s.write(total, [0] * len(lengths), k, v)
    q, out, lse = s.check_attend()
    assert (out == 0).all() and torch.isfinite(lse).all()


@pytest.mark.parametrize("lengths", [[1], [1] * 90, [3, 1], [70], [300, 1]])
@pytest.mark.parametrize("d,window", [(64, 40), (128, 200), (256, 100)])
@pytest.mark.parametrize("held", [500, 511, 512, 520, 543, 600])
def test_pages_behind_the_window_may_be_gone(lengths, d, window, held):
    """A server that frees the pages that a sliding window has left marks them as absent: nothing of a page that no row sees
    is asked for, wherever it lies in a step of the kernels."""
    from paper_2605_11222_b200 import adapt, kvcache
    s = Setup(lengths, [held] * len(lengths), 1, d, 16, seed=held, group=2)
    s.new_rows()
    q = torch.randn(sum(lengths), 2, d, generator=s.g, device=DEV).bfloat16()
    want = s.cache.attend(q, s.plan, window=window)
    adapt.check_device_status(DEV)
    first = (held - window + 1) // 16                        # the page of the first position that is seen
    for absent in (-1, 2 ** 30):
        gone = [[absent] * first + row[first:] for row in s.padded]
        out, lse = s.cache.attend(q, kvcache.CachePlan(lengths, s.held, gone, 2, DEV), window=window)
        adapt.check_device_status(DEV)
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
    # one page more is one that is seen
    gone = [[-1] * (first + 1) + row[first + 1:] for row in s.padded]
    s.cache.attend(q, kvcache.CachePlan(lengths, s.held, gone, 2, DEV), window=window)
    with pytest.raises(adapt.AdmmqError):
        adapt.check_device_status(DEV)


@pytest.mark.parametrize("sink", [0, 40, 100, 255, 1990])
@pytest.mark.parametrize("requests,rows,d", [(64, 1, 64), (64, 1, 128), (20, 70, 64), (20, 70, 128), (20, 70, 192)])
def test_weights_far_below_the_largest_of_their_row_are_kept(requests, rows, d, sink):
    """A token with nearly all of a row's weight and values of zero, in a block whose scale is that of the others: the
    result is what the others' weights make of it, 2^-25 to 2^-27 of the largest each, 2000 of them.  More (tile, head)s
    than CTAs, so that a CTA sees most of a row.

    Tolerance, beside the rounding of the result (2^-8 of it): a weight is rounded to fp16 with its row's largest at
    least 2^6 in the kernels' unit, so by 2^-12 of itself at most while it is above 2^-14, and below by half a step of 2^-24:
    2^-31 of the largest, at random: six standard deviations are 6 / sqrt(3) 2^-31 sqrt(sum v^2); the exponent of a weight (some 30) has
    2^-19 of error after a few roundings, the sums 2^-18: together 2^-17 sum w |v|."""
    from paper_2605_11222_b200 import adapt, kvcache
    heads, n, page = 8, 2000, 64
    g = _gen(d + rows)
    pages = -(-(n + rows) // page)
    cache = kvcache.KVCache(pages, heads, d, page, DEV)
    total = n + rows
    # one channel carries the score: that token's is 26 powers of two above the others', give or take one
    k, v = torch.zeros(total, heads, d, device=DEV), 0.5 + torch.rand(total, heads, d, generator=g, device=DEV)
    k[:, :, 0] = torch.rand(total, heads, generator=g, device=DEV)
    k[sink, :, 0] = 27.0
    v[sink] = 0.0
    cache.write(k.bfloat16(), v.bfloat16(), kvcache.CachePlan([total], [0], [list(range(pages))], device=DEV))
    q = torch.zeros(requests * rows, heads, d, device=DEV)
    q[..., 0] = 1.0
    plan = kvcache.CachePlan([rows] * requests, [n] * requests, [list(range(pages))] * requests, 1, DEV)   # all read the same pages
    out, lse = cache.attend(q.bfloat16(), plan, math.log(2.0))
    adapt.check_device_status(DEV)
    kk, vv = [x.double() for x in cache.read(kvcache.CachePlan([total], [0], [list(range(pages))], device=DEV), torch.float32)]
    z = kk[:, :, 0].T * math.log(2.0)                                                  # [heads, positions], of any row
    seen = torch.arange(total, device=DEV)[None] <= n + torch.arange(rows, device=DEV)[:, None]
    w = torch.softmax(z[:, None].masked_fill(~seen, -math.inf), -1)                    # [heads, rows, positions]
    assert (w[:, :, sink] > 0.99).all() and ((w < 2.0 ** -24).sum(-1) >= n - 1).all()
    want = torch.einsum("hrp,phd->rhd", w, vv)
    tiny = 6 / math.sqrt(3) * 2.0 ** -31 * (vv ** 2).sum(0).sqrt()                     # [heads, d]
    tol = 2.0 ** -8 * want.abs() + tiny + 2.0 ** -17 * torch.einsum("hrp,phd->rhd", w, vv.abs())
    lw = torch.logsumexp(z[:, None].masked_fill(~seen, -math.inf), -1).T
    for i in range(requests):
        _within(out[i * rows: (i + 1) * rows], want.cpu(), tol.cpu())
        _within(lse[i * rows: (i + 1) * rows], lw.cpu(), torch.full_like(lw, 2.0 ** -18 * 27).cpu())


@pytest.mark.parametrize("n", [1, 40, 100])
@pytest.mark.parametrize("size", [2.0 ** -133, 2.0 ** -126, 2.0 ** -115, 2.0 ** -110, 0.0])
def test_queries_near_zero(n, size):
    """A row of queries down to bf16's smallest numbers: its scores are zero as far as they matter, its weights equal."""
    s = Setup([n], [100], 2, 128, 64, group=2)
    s.new_rows()
    q = torch.randn(n, 4, 128, generator=s.g, device=DEV).bfloat16()
    q[0, 1] = size
    q[0, 2] = 0.0
    q[0, 2, 5] = -size
    s.check_attend(q=q)


def test_outputs_that_overlap_are_refused():
    from paper_2605_11222_b200 import adapt
    s = Setup([3, 2], [20, 0], 2, 64, 32, group=2)
    s.new_rows()
    q = torch.randn(5, 4, 64, generator=s.g, device=DEV).bfloat16()
    row = torch.zeros(5, 4, 64, dtype=torch.bfloat16, device=DEV)
    for bad in (row[:1].expand(5, 4, 64), row[:, :1].expand(5, 4, 64), row.as_strided((5, 4, 64), (64, 64, 1))):
        with pytest.raises(adapt.AdmmqError):
            s.cache.attend(q, s.plan, out=bad)
        with pytest.raises(adapt.AdmmqError):
            s.cache.read(s.plan, k=bad[:, :2])
        with pytest.raises(adapt.AdmmqError):
            s.cache.read(s.plan, v=bad[:, :2])
    want = s.cache.attend(q, s.plan)
    head_major = torch.zeros(4, 5, 64, dtype=torch.bfloat16, device=DEV).transpose(0, 1)
    got = s.cache.attend(q, s.plan, out=head_major)
    assert got[0] is head_major and torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    adapt.check_device_status(DEV)

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

"""GPU tests of the operators on quantized layers (adapt.py) against plain 64-bit formulas.

Tolerances, element by element, from the arithmetic (EPS = 2^-8 is half a bf16 ulp, relative: 8 significant bits):
 - an output rounded to bf16: EPS |result|;
 - operands rounded to bf16 inside a sum (weights expanded for the tensor cores, h and u of an expansion, factors of the
   adapters' gradients): independent errors of at most EPS |term| each, standard deviation at most EPS / sqrt(3) |term|,
   so six standard deviations are 6 EPS / sqrt(3) sqrt(sum term^2);
 - fp32 sums on the tensor cores, which may truncate: a step loses at most 2^-23 of the running sum, over at most 32 steps
   between folds (small kernel) or with errors that add up at random otherwise: 2^-18 sum |term|.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -8
SIX = 6.0 / math.sqrt(3.0)
ACC = 2.0 ** -18
DEV = "cuda:0"


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


def _layer(g, n, p, bits, group, sym=False):
    gs = group or n
    w = (_randn(g, p, n) * 0.02).view(p, n // gs, gs)
    lo, hi = w.amin(-1), w.amax(-1)
    if sym:
        hi = torch.maximum(hi, -lo)
        lo = -hi
    top = 2 ** bits - 1
    scale = (hi - lo) / top
    codes = torch.round((w - lo[..., None]) / scale[..., None]).clamp_(0, top).to(torch.uint8).view(p, n)
    return codes, scale.contiguous(), lo.contiguous()


def _weight64(codes, scale, zero):
    p, n = codes.shape
    gs = n // scale.shape[1]
    e = lambda t: t.double().repeat_interleave(gs, 1)  # noqa: E731
    return e(zero) + e(scale) * codes.double()


def _bank(g, na, r, n, p):
    from paper_2605_11222_b200 import adapt
    down = ((torch.rand(na, r, n, generator=g, device=DEV) * 2 - 1) / math.sqrt(n)).bfloat16()
    up = (_randn(g, na, r, p) * 0.02).bfloat16()
    return adapt.AdapterBank(down, up, torch.linspace(0.5, 2.0, na, device=DEV))


def _rows64(plan):
    a = plan.row_adapter.long()
    return a, (a >= 0).double()


def _shrink64(x, mat, bank, plan):
    """(values, sum of |term|)."""
    a, on = _rows64(plan)
    s = bank.scale.double()[a.clamp(min=0)] * on
    m = mat.double()[a.clamp(min=0)]
    x = x.double()
    return torch.einsum("ti,tri->tr", x, m) * s[:, None], torch.einsum("ti,tri->tr", x.abs(), m.abs()) * s[:, None]


def _expand64(u, mat, plan):
    """(values, sum of term^2)."""
    a, on = _rows64(plan)
    m = mat.double()[a.clamp(min=0)] * on[:, None, None]
    return torch.einsum("tr,tri->ti", u.double(), m), torch.einsum("tr,tri->ti", u.double() ** 2, m ** 2)


def _within(got, want, tol):
    err = (got.double() - want).abs()
    worst = (err / tol.clamp(min=1e-300)).max().item() if err.numel() else 0.0
    assert worst <= 1.0, f"error is {worst:.3g} of the tolerance"



def _plan(kind, T, na, seed=0):
    from paper_2605_11222_b200 import adapt
    g = torch.Generator().manual_seed(seed)
    if kind == "one":
        lengths, ids = [T], [na - 1]
    elif kind == "none":
        lengths, ids = [T], [-1]
    elif kind == "each":                         # a row a request, an adapter of its own as far as they go
        lengths, ids = [1] * T, [(5 * i) % (na + 1) - 1 for i in range(T)]
    else:                                        # ragged, some empty, some without an adapter
        cuts = torch.randint(0, T + 1, (5,), generator=g).sort().values.tolist()
        cuts = [0] + cuts[:3] + [cuts[2]] + cuts[3:] + [T]
        lengths = [b - a for a, b in zip(cuts, cuts[1:])]
        ids = torch.randint(-1, na, (len(lengths),), generator=g).tolist()
    return adapt.RequestPlan(lengths, ids, na)


# (rows, d_in, d_out, bits, group, symmetric, adapters, rank, plan)
LINEAR = [
    (1, 64, 8, 4, 64, False, 1, 8, "one"),
    (1, 4096, 1024, 4, 128, False, 3, 16, "one"),
    (2, 72, 40, 2, 0, True, 2, 8, "each"),
    (7, 512, 264, 3, 128, False, 4, 24, "each"),
    (8, 1000, 136, 4, 0, False, 5, 32, "mixed"),
    (9, 4096, 1024, 2, 0, True, 16, 8, "each"),
    (16, 576, 1000, 4, 64, False, 3, 128, "mixed"),
    (17, 576, 1000, 4, 64, False, 3, 128, "mixed"),
    (33, 8, 8, 4, 0, False, 2, 8, "mixed"),
    (64, 256, 384, 3, 128, True, 6, 16, "each"),
    (65, 1024, 128, 4, 256, False, 2, 48, "mixed"),
    (128, 200, 136, 2, 0, False, 40, 8, "each"),
    (129, 4096, 520, 4, 128, False, 4, 64, "mixed"),
    (4, 4096, 40, 3, 128, False, 3, 8, "each"),         # one launch, input channels split
    (1, 14336, 24, 4, 64, False, 2, 32, "one"),
    (5, 2048, 8200, 4, 64, False, 3, 56, "each"),       # two launches
    (16, 14336, 16, 4, 256, False, 3, 16, "each"),
    (16, 1032, 8192, 2, 0, True, 6, 16, "each"),
    (300, 1344, 1096, 3, 64, False, 70, 8, "each"),
    (520, 768, 2056, 4, 128, True, 3, 72, "none"),
    (1030, 2048, 392, 4, 0, False, 3, 16, "mixed"),
]


@pytest.mark.parametrize("T,n,p,bits,group,sym,na,r,kind", LINEAR)
def test_forward_matches_the_formula(T, n, p, bits, group, sym, na, r, kind):
    from paper_2605_11222_b200 import adapt
    g = _gen(T + n)
    codes, scale, zero = _layer(g, n, p, bits, group, sym)
    layer = adapt.QuantLinear(codes, scale, zero, bits, group)
    bank, plan = _bank(g, na, r, n, p), _plan(kind, T, na, T)
    x = _randn(g, T, n)
    x[:, :: 97] *= 30.0                          # outlier channels
    x = x.bfloat16()
    y, h = layer.forward(x, bank, plan)
    adapt.check_device_status(DEV)
    W = _weight64(codes, scale, zero)
    want_h, abs_h = _shrink64(x, bank.down, bank, plan)
    _within(h, want_h, ACC * abs_h + 1e-30)
    base = x.double() @ W.T
    delta, sq_delta = _expand64(want_h, bank.up, plan)
    want = base + delta
    sq = x.double() ** 2 @ (W ** 2).T + sq_delta
    top = scale.double().amax(1) * 143 + zero.double().abs().amax(1)      # 128 + k steps of the grid, and its origin
    acc = ACC * (x.double().abs().sum(1)[:, None] * top[None] + sq_delta.sqrt() * math.sqrt(r))
    rounding = torch.zeros_like(want) if T <= 16 else SIX * EPS * sq.sqrt()
    _within(y, want, EPS * want.abs() + acc + rounding + 1e-30)
    # without adapters
    y0, h0 = layer.forward(x)
    assert h0 is None
    _within(y0, base, EPS * base.abs() + acc + rounding + 1e-30)


@pytest.mark.parametrize("T,n,p,bits,group,sym,na,r,kind", LINEAR)
def test_grad_input_matches_the_formula(T, n, p, bits, group, sym, na, r, kind):
    from paper_2605_11222_b200 import adapt
    g = _gen(T + p)
    codes, scale, zero = _layer(g, n, p, bits, group, sym)
    layer = adapt.QuantLinear(codes, scale, zero, bits, group)
    bank, plan = _bank(g, na, r, n, p), _plan(kind, T, na, T)
    dy = (_randn(g, T, p) * 1e-3).bfloat16()
    dx, u = layer.grad_input(dy, bank, plan)
    adapt.check_device_status(DEV)
    W = _weight64(codes, scale, zero)
    want_u, abs_u = _shrink64(dy, bank.up, bank, plan)
    _within(u, want_u, ACC * abs_u + 1e-30)
    base = dy.double() @ W
    delta, sq_delta = _expand64(want_u, bank.down, plan)
    want = base + delta
    sq = dy.double() ** 2 @ W ** 2 + sq_delta
    acc = ACC * (dy.double().abs() @ W.abs() + sq_delta.sqrt() * math.sqrt(r))
    _within(dx, want, EPS * want.abs() + SIX * EPS * sq.sqrt() + acc + 1e-30)
    dx0, _ = layer.grad_input(dy)
    _within(dx0, base, EPS * base.abs() + SIX * EPS * sq.sqrt() + acc + 1e-30)


# (rows, d_in, d_out, adapters, rank, plan, checkpoint)
GRADS = [
    (0, 64, 64, 2, 8, "none", True), (1, 136, 8, 1, 8, "one", True), (5, 128, 264, 3, 16, "mixed", False),
    (63, 1000, 128, 2, 24, "mixed", True), (64, 256, 384, 4, 32, "each", True), (65, 256, 384, 70, 8, "each", False),
    (333, 4096, 1024, 3, 64, "mixed", True), (1500, 392, 520, 1, 128, "one", True), (4100, 264, 200, 2, 16, "mixed", False),
    (200, 72, 136, 2, 48, "none", True),
]


@pytest.mark.parametrize("T,n,p,na,r,kind,eight", GRADS)
def test_adapter_grads_match_the_formula(T, n, p, na, r, kind, eight):
    from paper_2605_11222_b200 import adapt
    g = _gen(T * 3 + n)
    bank, plan = _bank(g, na, r, n, p), _plan(kind, T, na, T)
    x = _randn(g, T, n).bfloat16()
    dy = (_randn(g, T, p) * 1e-3).bfloat16()
    h, u = _randn(g, T, r), _randn(g, T, r) * 1e-3
    v = x
    x64 = x.double()
    if eight:
        v = adapt.Checkpoint.save(x)
        x64 = v.codes.double() * v.scale.double().repeat_interleave(128, 1)[:, :n]
    d_down, d_up = adapt.adapter_grads(bank, plan, v, h, dy, u)
    for a in range(na):
        t = (plan.row_adapter == a).nonzero()[:, 0]
        for got, f, w in ((d_down[a], u, x64), (d_up[a], h, dy.double())):
            want = f[t].double().T @ w[t]
            sq, ab = (f[t].double() ** 2).T @ w[t] ** 2, f[t].double().abs().T @ w[t].abs()
            _within(got, want, EPS * want.abs() + SIX * EPS * sq.sqrt() + ACC * ab + 1e-30)


# tiles of one CTA with and without a split of K, and tiles of CTA pairs (many rows); K of few and of many steps
@pytest.mark.parametrize("T,n,p,na,r", [(70, 512, 256, 2, 8), (200, 4096, 512, 3, 24), (600, 512, 256, 2, 8),
                                        (3000, 1024, 2048, 2, 8), (2600, 192, 4096, 5, 72), (2600, 4096, 64, 40, 16),
                                        (9000, 256, 1024, 3, 48)])
def test_projections_are_the_same_bits_every_time(T, n, p, na, r):
    """The order of every sum is fixed, so a difference between two runs is a race.  Other shapes than the formula tests'
    (more rows, so that multiprocessors work on several tiles), checked against the formula row by row as well."""
    from paper_2605_11222_b200 import adapt
    g = _gen(T)
    codes, scale, zero = _layer(g, n, p, 4, 64)
    layer, bank, plan = adapt.QuantLinear(codes, scale, zero, 4, 64), _bank(g, na, r, n, p), _plan("mixed", T, na, 5)
    x, dy = _randn(g, T, n).bfloat16(), _randn(g, T, p).bfloat16()
    W = _weight64(codes, scale, zero)
    for run, v, w, inn, out in ((layer.forward, x, W.T, bank.down, bank.up), (layer.grad_input, dy, W, bank.up, bank.down)):
        first = run(v, bank, plan)
        f64 = torch.zeros(T, r, dtype=torch.float64, device=DEV)
        want, sq = v.double() @ w, v.double() ** 2 @ w ** 2
        for a in range(na):
            t = (plan.row_adapter == a).nonzero()[:, 0]
            f64[t] = bank.scale[a].double() * (v[t].double() @ inn[a].double().T)
            want[t] += f64[t] @ out[a].double()
            sq[t] += f64[t] ** 2 @ out[a].double() ** 2
        _within(first[0], want, EPS * want.abs() + SIX * EPS * sq.sqrt() + ACC * sq.sqrt() * math.sqrt(w.shape[0]) + 1e-30)
        for _ in range(40):
            again = run(v, bank, plan)
            assert torch.equal(again[0], first[0]) and torch.equal(again[1], first[1])
    adapt.check_device_status(DEV)


@pytest.mark.parametrize("k", [64, 192, 576])                # contracted channels: one, three and nine K steps
@pytest.mark.parametrize("r", [24, 64, 128])                 # two adapters in a K step, one, half of one
def test_pairs_with_several_tiles_and_changing_numbers_of_adapters(k, r):
    """216 tiles of 512 rows and 256 values, so that every pair of multiprocessors has two or three, from one to the next
    with another number of adapter steps (0 to 5 adapters in 512 rows)."""
    from paper_2605_11222_b200 import adapt
    T, m, na = 24 * 512, 2304, 6
    g = _gen(k + r)
    lengths, ids = [], []
    for tile in range(24):
        n = (5 * tile + tile // 6) % 6                         # distinct adapters of the tile
        for i in range(max(1, n)):
            lengths.append(512 // max(1, n) if i else 512 - 512 // max(1, n) * (max(1, n) - 1))
            ids.append((tile + i) % na if n else -1)
    plan = adapt.RequestPlan(lengths, ids, na)
    assert plan.n_rows == T
    for grad in (False, True):
        n, p = (m, k) if grad else (k, m)
        codes, scale, zero = _layer(g, n, p, 4, 64)
        layer, bank = adapt.QuantLinear(codes, scale, zero, 4, 64), _bank(g, na, r, n, p)
        W = _weight64(codes, scale, zero)
        v = _randn(g, T, k).bfloat16()
        run, w, inn, out = (layer.grad_input, W, bank.up, bank.down) if grad else (layer.forward, W.T, bank.down, bank.up)
        first = run(v, bank, plan)
        want, sq = v.double() @ w, v.double() ** 2 @ w ** 2
        for a in range(na):
            t = (plan.row_adapter == a).nonzero()[:, 0]
            f64 = bank.scale[a].double() * (v[t].double() @ inn[a].double().T)
            want[t] += f64 @ out[a].double()
            sq[t] += f64 ** 2 @ out[a].double() ** 2
        _within(first[0], want, EPS * want.abs() + SIX * EPS * sq.sqrt() + ACC * sq.sqrt() * math.sqrt(k + r) + 1e-30)
        for _ in range(30):
            assert torch.equal(run(v, bank, plan)[0], first[0])
        # without a bank
        want, sq = v.double() @ w, v.double() ** 2 @ w ** 2
        _within(run(v)[0], want, EPS * want.abs() + SIX * EPS * sq.sqrt() + ACC * sq.sqrt() * math.sqrt(k) + 1e-30)
        adapt.check_device_status(DEV)


@pytest.mark.parametrize("r", [8, 16, 24, 32])
@pytest.mark.parametrize("T", [70, 300])
def test_adapters_of_a_tile_in_runs_and_with_gaps(T, r):
    from paper_2605_11222_b200 import adapt
    g = _gen(T + r)
    n, p, na = 256, 200, 12
    codes, scale, zero = _layer(g, n, p, 4, 64)
    layer, bank = adapt.QuantLinear(codes, scale, zero, 4, 64), _bank(g, na, r, n, p)
    W = _weight64(codes, scale, zero)
    x, dy = _randn(g, T, n).bfloat16(), _randn(g, T, p).bfloat16()
    for ids in ([0, 1, 2, 3], [4, 5, 6, 7, 8, 9, 10, 11], [11, 9, 10], [0, 2, 3, 7, 8, 11], [5, -1, 6], list(range(na))):
        cuts = [T * i // len(ids) for i in range(len(ids) + 1)]
        plan = adapt.RequestPlan([b - a for a, b in zip(cuts, cuts[1:])], ids, na)
        for run, v, w, inn, out in ((layer.forward, x, W.T, bank.down, bank.up), (layer.grad_input, dy, W, bank.up, bank.down)):
            y, _ = run(v, bank, plan)
            h, _ = _shrink64(v, inn, bank, plan)
            delta, sq_delta = _expand64(h, out, plan)
            want, sq = v.double() @ w + delta, v.double() ** 2 @ w ** 2 + sq_delta
            _within(y, want, EPS * want.abs() + SIX * EPS * sq.sqrt() + ACC * sq.sqrt() * math.sqrt(w.shape[0] + r) + 1e-30)
    adapt.check_device_status(DEV)


# (rows, contracted channels, adapters, rank, plan): stacked adapters that fit a pass and that do not, ranks that leave
# lanes over, channels that end inside a step, tiles past the rows, contracted channels split over several blocks
CONTRACTIONS = [
    (256, 8, 1, 128, "one"),
    (257, 1000, 3, 128, "each"),
    (512, 128, 2, 64, "none"),
    (600, 576, 12, 64, "each"),
    (1024, 200, 3, 32, "mixed"),
    (1100, 4096, 2, 32, "one"),
    (1400, 72, 5, 24, "mixed"),
    (4097, 136, 20, 8, "each"),
    (4200, 520, 3, 16, "mixed"),
    (5000, 264, 2, 40, "mixed"),
    (4500, 2048, 9, 16, "each"),
]


@pytest.mark.parametrize("T,n,na,r,kind", CONTRACTIONS)
def test_contraction_of_many_rows(T, n, na, r, kind):
    from paper_2605_11222_b200 import adapt
    g = _gen(T + n)
    codes, scale, zero = _layer(g, n, 8, 4, 0)
    back = _layer(g, 8, n, 4, 0)
    bank, turned = _bank(g, na, r, n, 8), _bank(g, na, r, 8, n)
    plan = _plan(kind, T, na, T)
    x = _randn(g, T, n + 8).bfloat16()[:, :n]     # rows that are not adjacent
    for layer, b, mat, run in ((adapt.QuantLinear(codes, scale, zero, 4, 0), bank, bank.down, "forward"),
                               (adapt.QuantLinear(*back, 4, 0), turned, turned.up, "grad_input")):
        _, h = getattr(layer, run)(x, b, plan)
        adapt.check_device_status(DEV)
        for t in range(0, T, 1000):               # (the plain form gathers a matrix a row)
            rows = slice(t, min(T, t + 1000))

            class Part:
                row_adapter = plan.row_adapter[rows]
            want, size = _shrink64(x[rows], mat, b, Part)
            _within(h[rows], want, ACC * size + 1e-30)
        for _ in range(10):
            assert torch.equal(getattr(layer, run)(x, b, plan)[1], h)


def test_a_bad_row_stays_in_its_row_of_the_contraction():
    from paper_2605_11222_b200 import adapt
    g = _gen(31)
    codes, scale, zero = _layer(g, 512, 8, 4, 128)
    layer, bank, plan = adapt.QuantLinear(codes, scale, zero, 4, 128), _bank(g, 3, 64, 512, 8), _plan("each", 700, 3)
    x = _randn(g, 700, 512).bfloat16()
    _, want = layer.forward(x, bank, plan)
    x[333, 5] = float("nan")
    x[12, 7] = float("inf")
    _, h = layer.forward(x, bank, plan)
    keep = torch.ones(700, dtype=torch.bool, device=DEV)
    keep[[12, 333]] = False
    assert torch.equal(h[keep], want[keep])
    on = (plan.row_adapter[[12, 333]] >= 0)
    assert not torch.isfinite(h[[12, 333]][on]).any() and (h[[12, 333]][~on] == 0).all()


def test_a_wait_of_the_contraction_that_runs_out_is_reported():
    from paper_2605_11222_b200 import adapt, binding as B
    g = _gen(3)
    codes, scale, zero = _layer(g, 1024, 256, 4, 128)
    layer, bank, plan = adapt.QuantLinear(codes, scale, zero, 4, 128), _bank(g, 3, 64, 1024, 256), _plan("each", 600, 3)
    x = _randn(g, 600, 1024).bfloat16()
    want, wanth = layer.forward(x, bank, plan)
    lib = adapt._library()
    assert lib.admmq_test_linear_set_wait(200000, 1) == B.OK
    try:
        layer.forward(x, bank, plan)
        with pytest.raises(adapt.AdmmqError) as e:
            adapt.check_device_status(DEV)
        assert e.value.status == B.ERR_TIMEOUT
    finally:
        assert lib.admmq_test_linear_set_wait(2_000_000_000, 0) == B.OK
    got, h = layer.forward(x, bank, plan)
    adapt.check_device_status(DEV)
    assert torch.equal(got, want) and torch.equal(h, wanth)


@pytest.mark.parametrize("T,n,p,r", [(1, 64, 72, 8), (70, 264, 128, 24), (900, 512, 392, 64)])
def test_adapter_grads_of_strided_rows_into_given_tensors(T, n, p, r):
    from paper_2605_11222_b200 import adapt
    g = _gen(T + r)
    bank, plan = _bank(g, 3, r, n, p), _plan("mixed", T, 3, 1)
    x, dy = _randn(g, T, n + 40).bfloat16(), (_randn(g, T, p + 8) * 1e-3).bfloat16()
    h, u = _randn(g, T, r), _randn(g, T, r) * 1e-3
    xs, dys = x[:, 16:16 + n], dy[:, 8:]
    for v, dense in ((xs, xs.contiguous()), (adapt.Checkpoint.save(xs), adapt.Checkpoint.save(xs.contiguous()))):
        want = adapt.adapter_grads(bank, plan, dense, h, dys.contiguous(), u)
        got = adapt.adapter_grads(bank, plan, v, h, dys, u)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        gd, gu = torch.full_like(bank.down, 9.0), torch.full_like(bank.up, 9.0)
        for given in (dict(grad_down=gd, grad_up=gu), dict(grad_down=gd), dict(grad_up=gu)):
            got = adapt.adapter_grads(bank, plan, v, h, dys, u, **given)
            assert all(torch.equal(a, b) for a, b in zip(got, want))
            assert got[0] is given.get("grad_down", got[0]) and got[1] is given.get("grad_up", got[1])


def test_adapter_grads_are_the_same_bits_every_time():
    from paper_2605_11222_b200 import adapt
    g = _gen(9)
    bank, plan = _bank(g, 2, 16, 512, 256), _plan("mixed", 3000, 2, 4)
    x, dy = _randn(g, 3000, 512).bfloat16(), _randn(g, 3000, 256).bfloat16()
    h, u = _randn(g, 3000, 16), _randn(g, 3000, 16)
    first = adapt.adapter_grads(bank, plan, x, h, dy, u)
    for _ in range(3):
        again = adapt.adapter_grads(bank, plan, x, h, dy, u)
        assert all(torch.equal(a, b) for a, b in zip(first, again))


@pytest.mark.parametrize("T", [11, 150, 13000])
def test_gradients_agree_with_differences(T):
    """The output is linear in x and in each adapter matrix, so a difference over any step is the derivative; what is left
    is the rounding of the outputs to bf16, EPS |y| each with independent signs."""
    from paper_2605_11222_b200 import adapt
    n, p, na, r = 512, 384, 2, 16
    g = _gen(T)
    codes, scale, zero = _layer(g, n, p, 4, 128)
    layer, bank, plan = adapt.QuantLinear(codes, scale, zero, 4, 128), _bank(g, na, r, n, p), _plan("mixed", T, na, 3)
    x, dy = _randn(g, T, n).bfloat16(), _randn(g, T, p).bfloat16()
    y, h = layer.forward(x, bank, plan)
    dx, u = layer.grad_input(dy, bank, plan)
    d_down, d_up = adapt.adapter_grads(bank, plan, x, h, dy, u)

    def loss(x, down, up):
        out, _ = layer.forward(x, adapt.AdapterBank(down, up, bank.scale), plan)
        return out.double()

    for name, grad, value in (("x", dx, x), ("down", d_down, bank.down), ("up", d_up, bank.up)):
        step = _randn(g, *value.shape).bfloat16() if name == "x" else (value * 4).bfloat16()
        at = {"x": x, "down": bank.down, "up": bank.up}
        hi, lo = dict(at), dict(at)
        hi[name], lo[name] = (value + step).bfloat16(), (value - step).bfloat16()
        moved = hi[name].double() - lo[name].double()              # what the step is after rounding
        yh, yl = loss(**hi), loss(**lo)
        got = ((yh - yl) * dy.double()).sum()
        want = (grad.double() * moved).sum()
        # roundings: both outputs (and their weights), and the gradient's own entries
        noise = 2 * SIX * EPS * (((yh.abs() + yl.abs() + 1) * dy.double()) ** 2).sum().sqrt() \
            + 2 * SIX * EPS * ((grad.double() * moved) ** 2).sum().sqrt()
        assert abs(got - want) <= noise, (name, float(got), float(want), float(noise))


@pytest.mark.parametrize("T", [9, 37, 20000])                  # one form of the projection each
def test_strided_rows_outputs_and_another_stream(T):
    from paper_2605_11222_b200 import adapt
    g = _gen(5)
    n, p = 256, 136
    codes, scale, zero = _layer(g, n, p, 3, 64)
    layer, bank, plan = adapt.QuantLinear(codes, scale, zero, 3, 64), _bank(g, 2, 8, n, p), _plan("mixed", T, 2, 1)
    big = _randn(g, T, n + 24).bfloat16()
    x = big[:, 16: 16 + n]
    out = torch.full((T, p + 8), 7.0, dtype=torch.bfloat16, device=DEV)
    y, h = layer.forward(x, bank, plan)
    layer.forward(x, bank, plan, out=out[:, :p])
    assert torch.equal(out[:, :p], y) and bool((out[:, p:] == 7).all())
    dx = torch.full((T, n + 8), 7.0, dtype=torch.bfloat16, device=DEV)
    ref, _ = layer.grad_input(y, bank, plan)
    layer.grad_input(out[:, :p], bank, plan, out=dx[:, :n])
    assert torch.equal(dx[:, :n], ref) and bool((dx[:, n:] == 7).all())
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        y2, h2 = layer.forward(x, bank, plan)
    s.synchronize()
    assert torch.equal(y, y2) and torch.equal(h, h2)


@pytest.mark.parametrize("T", [5, 40, 20000])
def test_forward_in_a_cuda_graph(T):
    from paper_2605_11222_b200 import adapt
    g = _gen(6)
    n, p = 512, 256
    codes, scale, zero = _layer(g, n, p, 4, 128)
    layer, bank, plan = adapt.QuantLinear(codes, scale, zero, 4, 128), _bank(g, 3, 16, n, p), _plan("each", T, 3)
    x = _randn(g, T, n).bfloat16()
    y, h = torch.empty(T, p, dtype=torch.bfloat16, device=DEV), torch.empty(T, 16, device=DEV)
    layer.forward(x, bank, plan, out=y, h=h)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.forward(x, bank, plan, out=y, h=h)
    x.copy_(_randn(g, T, n))
    graph.replay()
    want, _ = layer.forward(x, bank, plan)
    torch.cuda.synchronize()
    assert torch.equal(y, want)


@pytest.mark.parametrize("T", [6, 50, 40000])
def test_a_bad_row_stays_in_its_row(T):
    """A NaN or infinity in one row's input does not reach another row, whatever adapters they have."""
    from paper_2605_11222_b200 import adapt
    g = _gen(8)
    n, p = 256, 128
    codes, scale, zero = _layer(g, n, p, 4, 64)
    layer, bank, plan = adapt.QuantLinear(codes, scale, zero, 4, 64), _bank(g, 3, 8, n, p), _plan("each", T, 3)
    x = _randn(g, T, n).bfloat16()
    want, _ = layer.forward(x, bank, plan)
    bad = x.clone()
    bad[1, 3], bad[4, 9] = float("nan"), float("inf")
    got, _ = layer.forward(bad, bank, plan)
    keep = [t for t in range(T) if t not in (1, 4)]
    assert torch.equal(got[keep], want[keep])
    assert not torch.isfinite(got[1].float()).any() and not torch.isfinite(got[4].float()).any()


def test_a_bank_with_a_non_finite_entry_is_refused():
    from paper_2605_11222_b200 import adapt, binding as B
    g = _gen(10)
    bank = _bank(g, 2, 8, 64, 64)
    for t, bad in ((bank.down, float("inf")), (bank.up, float("nan"))):
        keep = t[1, 7, 63].clone()
        t[1, 7, 63] = bad
        with pytest.raises(adapt.AdmmqError) as e:
            bank.check()
        assert e.value.status == B.ERR_NONFINITE
        t[1, 7, 63] = keep
        bank.check()


def test_codes_beyond_the_bits_are_refused():
    from paper_2605_11222_b200 import adapt, binding as B
    codes, scale, zero = _layer(_gen(1), 64, 8, 3, 0)
    codes[5, 60] = 8
    with pytest.raises(adapt.AdmmqError) as e:
        adapt.QuantLinear(codes, scale, zero, 3)
    assert e.value.status == B.ERR_INVALID_ARG
    adapt.QuantLinear(codes, scale, zero, 4)


def test_refusals():
    from paper_2605_11222_b200 import adapt, binding as B
    g = _gen(2)
    codes, scale, zero = _layer(g, 128, 64, 4, 64)
    layer, bank, plan = adapt.QuantLinear(codes, scale, zero, 4, 64), _bank(g, 2, 8, 128, 64), _plan("mixed", 9, 2)
    x = _randn(g, 9, 128).bfloat16()

    def refused(status, f, *a, **k):
        with pytest.raises(adapt.AdmmqError) as e:
            f(*a, **k)
        assert e.value.status == status

    refused(B.ERR_UNSUPPORTED, adapt.QuantLinear, codes, scale, zero, 5, 64)
    refused(B.ERR_SHAPE, adapt.QuantLinear, codes, scale, zero, 1, 64)
    refused(B.ERR_SHAPE, adapt.QuantLinear, codes, scale, zero, 4, 32)          # 4 groups: wrong count of scales
    c2, s2, z2 = _layer(g, 128, 64, 4, 32)
    refused(B.ERR_SHAPE, adapt.QuantLinear, c2, s2, z2, 4, 32)                   # a group of 32
    refused(B.ERR_INVALID_ARG, adapt.QuantLinear, codes.int(), scale, zero, 4, 64)
    refused(B.ERR_INVALID_ARG, layer.forward, x.float(), bank, plan)
    refused(B.ERR_SHAPE, layer.forward, x[:, :120], bank, plan)
    refused(B.ERR_SHAPE, layer.forward, x[:8], bank, plan)                       # another number of rows
    refused(B.ERR_SHAPE, layer.forward, x, bank)                                 # a bank without a plan
    odd = torch.empty(9, 132, dtype=torch.bfloat16, device=DEV)
    refused(B.ERR_SHAPE, layer.forward, odd[:, :128])                            # rows of 264 bytes
    refused(B.ERR_INVALID_ARG, layer.forward, torch.empty(9 * 136, dtype=torch.bfloat16, device=DEV)[1:1 + 8 * 136 + 128]
            .as_strided((9, 128), (136, 1)))                                     # not on a 16-byte boundary
    refused(B.ERR_SHAPE, adapt.RequestPlan, [1, -1], [0, 0], 2)
    refused(B.ERR_INVALID_ARG, adapt.RequestPlan, [1], [2], 2)
    h = torch.zeros(9, 8, device=DEV)
    y = torch.zeros(9, 64, dtype=torch.bfloat16, device=DEV)
    refused(B.ERR_SHAPE, adapt.adapter_grads, bank, plan, x, h[:8], y, h)
    refused(B.ERR_SHAPE, adapt.Checkpoint.save, torch.zeros(3, 12, device=DEV))
    refused(B.ERR_INVALID_ARG, adapt.Checkpoint.save, torch.zeros(3, 16, device=DEV).half())
    adapt.check_device_status(DEV)
    e = layer.forward(x[:0])[0]
    assert e.shape == (0, 64)


def test_a_wait_that_runs_out_is_reported():
    """The producer withholds its loads, so the first wait of every CTA expires with nothing in flight."""
    from paper_2605_11222_b200 import adapt, binding as B
    g = _gen(3)
    codes, scale, zero = _layer(g, 512, 256, 4, 128)
    layer, bank, plan = adapt.QuantLinear(codes, scale, zero, 4, 128), _bank(g, 2, 8, 512, 256), _plan("mixed", 70, 2)
    x = _randn(g, 70, 512).bfloat16()
    want, _ = layer.forward(x, bank, plan)
    lib = adapt._library()
    assert lib.admmq_test_linear_set_wait(10, 0) == B.ERR_INVALID_ARG
    assert lib.admmq_test_linear_set_wait(200000, 1) == B.OK
    try:
        layer.forward(x, bank, plan)
        with pytest.raises(adapt.AdmmqError) as e:
            adapt.check_device_status(DEV)
        assert e.value.status == B.ERR_TIMEOUT
    finally:
        assert lib.admmq_test_linear_set_wait(2_000_000_000, 0) == B.OK
    got, _ = layer.forward(x, bank, plan)
    adapt.check_device_status(DEV)
    assert torch.equal(got, want)


# one CTA a tile with K split over a cluster, one without, pairs with one tile each, pairs with several
@pytest.mark.parametrize("grad", [False, True])
@pytest.mark.parametrize("T,n,p,r", [(200, 4096, 512, 24), (900, 4096, 4096, 8), (20000, 256, 136, 16), (40000, 256, 392, 72)])
def test_a_wait_that_runs_out_is_reported_in_every_form_and_direction(T, n, p, r, grad):
    from paper_2605_11222_b200 import adapt, binding as B
    g = _gen(T + r)
    codes, scale, zero = _layer(g, n, p, 4, 64)
    layer, bank, plan = adapt.QuantLinear(codes, scale, zero, 4, 64), _bank(g, 3, r, n, p), _plan("mixed", T, 3, 2)
    run, v = (layer.grad_input, _randn(g, T, p).bfloat16()) if grad else (layer.forward, _randn(g, T, n).bfloat16())
    want = run(v, bank, plan), run(v)
    adapt.check_device_status(DEV)
    lib = adapt._library()
    for args in ((v, bank, plan), (v,)):
        assert lib.admmq_test_linear_set_wait(200000, 1) == B.OK
        try:
            run(*args)
            with pytest.raises(adapt.AdmmqError) as e:
                adapt.check_device_status(DEV)
            assert e.value.status == B.ERR_TIMEOUT
        finally:
            assert lib.admmq_test_linear_set_wait(2_000_000_000, 0) == B.OK
        assert torch.equal(run(v, bank, plan)[0], want[0][0]) and torch.equal(run(v)[0], want[1][0])
        adapt.check_device_status(DEV)


def test_a_whole_warp_wait_gives_every_lane_the_same_answer():
    """Also where some lanes give up before the barrier completes and the others would have seen it complete: the roles of
    the projections go on to warp-wide instructions by this answer."""
    from paper_2605_11222_b200 import adapt, binding as B
    lib = adapt._library()
    out = torch.full((32,), 7, dtype=torch.int32, device=DEV)
    long, short = 1_000_000_000, 20_000
    for low, high, answer in ((long, long, 1), (short, long, 0), (long, short, 0), (short, short, 0)):
        word = torch.zeros(1, dtype=torch.int32, device=DEV)
        assert lib.admmq_test_warp_wait(low, high, out.data_ptr(), word.data_ptr(),
                                        torch.cuda.current_stream().cuda_stream) == B.OK
        assert out.tolist() == [answer] * 32
        assert int(word) == (B.OK if answer else B.ERR_TIMEOUT)


@pytest.mark.parametrize("T,p", [(1, 64), (5, 136), (16, 200), (12, 8200)])
@pytest.mark.parametrize("n,group", [(64, 0), (512, 128), (4096, 0)])
def test_few_rows_keep_sums_that_fp32_holds(T, p, n, group):
    """Whole numbers: Delta = 1, z0 = -8, and in every 64 input channels two of 2^17 or -2^17 with the code 8 (weight 0)
    beside sixteen of 1 to 3 and zeros.  The terms (16 + k) x of the 64, and the sums of them, stay below 2^23 (24 * 2^18
    + 31 * 48), as do those of sum x times z0 - 16 Delta = -24, so every step is exact and the result, a whole number of at
    most 8 * 48 * blocks, is too; it is rounded once, to bf16."""
    from paper_2605_11222_b200 import adapt
    g = _gen(T + n)
    blocks = n // 64
    codes = torch.randint(0, 16, (p, n), generator=g, device=DEV, dtype=torch.uint8)
    x = torch.zeros(T, n, device=DEV)
    for b in range(blocks):
        at = torch.randperm(64, generator=g, device=DEV) + 64 * b
        sign = torch.randint(0, 2, (T, 1), generator=g, device=DEV) * 2 - 1
        x[:, at[:2]] = 2.0 ** 17 * sign
        codes[:, at[:2]] = 8
        x[:, at[2:18]] = torch.randint(1, 4, (T, 16), generator=g, device=DEV).float()
    groups = n // (group or n)
    scale, zero = torch.ones(p, groups, device=DEV), torch.full((p, groups), -8.0, device=DEV)
    y, _ = adapt.QuantLinear(codes, scale, zero, 4, group).forward(x.bfloat16())
    assert torch.equal(x.bfloat16().float(), x)
    want = x.double() @ (codes.double() - 8).T
    assert torch.equal(y, want.float().bfloat16())


@pytest.mark.parametrize("which", ["down", "up", "scale"])
def test_a_bank_whose_tensor_has_other_storage_is_refused(which):
    """The bank holds the addresses: with another storage behind the tensor they may be anyone's memory."""
    from paper_2605_11222_b200 import adapt, binding as B
    g = _gen(44)
    codes, scale, zero = _layer(g, 128, 64, 4, 64)
    layer, bank, plan = adapt.QuantLinear(codes, scale, zero, 4, 64), _bank(g, 2, 8, 128, 64), _plan("mixed", 9, 2)
    x, out = _randn(g, 9, 128).bfloat16(), torch.empty(9, 64, dtype=torch.bfloat16, device=DEV)
    layer.forward(x, bank, plan)
    t = getattr(bank, which)
    old = t.detach()                              # (keeps the old storage)
    t.data = t.clone()
    for call in (lambda: layer.forward(x, bank, plan), lambda: layer.forward(x, bank, plan, out=out),
                 lambda: layer.grad_input(out, bank, plan), bank.check):
        with pytest.raises(adapt.AdmmqError, match="storage") as e:
            call()
        assert e.value.status == B.ERR_INVALID_ARG
    new = adapt.AdapterBank(bank.down, bank.up, bank.scale)
    assert torch.isfinite(layer.forward(x, new, plan)[0].float()).all() and old.data_ptr() != t.data_ptr()


def _leave_an_error(adapt):
    """A call whose error stays in the device's status word: a position past the table."""
    q, w = torch.ones(1, 1, 16, device=DEV), torch.ones(16, device=DEV)
    cos, pos = torch.ones(2, 8, device=DEV), torch.full((1,), 2, dtype=torch.int32, device=DEV)
    adapt.qk_norm_rope(q, q, w, w, cos, cos, pos)


def test_a_sound_layer_and_bank_do_not_meet_another_calls_error():
    from paper_2605_11222_b200 import adapt, binding as B
    g = _gen(41)
    codes, scale, zero = _layer(g, 128, 64, 4, 64)
    adapt.check_device_status(DEV)
    _leave_an_error(adapt)
    adapt.QuantLinear(codes, scale, zero, 4, 64)
    _bank(g, 2, 8, 128, 64).check()
    with pytest.raises(adapt.AdmmqError) as e:                       # and the error is still there
        adapt.check_device_status(DEV)
    assert e.value.status == B.ERR_SHAPE
    adapt.check_device_status(DEV)


def test_threads_do_not_take_each_others_errors():
    import threading
    from paper_2605_11222_b200 import adapt, binding as B
    codes, scale, zero = _layer(_gen(42), 64, 8, 3, 0)
    codes[5, 60] = 8
    adapt.check_device_status(DEV)
    seen, stop = [], threading.Event()

    def packs():
        for _ in range(200):
            try:
                adapt.QuantLinear(codes, scale, zero, 3)
                seen.append(B.OK)
            except adapt.AdmmqError as e:
                seen.append(e.status)
        stop.set()

    def checks():
        while not stop.is_set():
            try:
                adapt.check_device_status(DEV)
            except adapt.AdmmqError as e:
                seen.append(e.status)

    threads = [threading.Thread(target=f) for f in (packs, checks)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert seen == [B.ERR_INVALID_ARG] * 200


def test_status_word_made_and_cleared_in_different_modes():
    from paper_2605_11222_b200 import adapt
    adapt.check_device_status(DEV)
    kept = dict(adapt._status_words)             # (calls hold the pointer of the word that was there)
    try:
        adapt._status_words.clear()
        with torch.inference_mode():
            _leave_an_error(adapt)
        with pytest.raises(adapt.AdmmqError):
            adapt.check_device_status(DEV)
    finally:
        adapt._status_words.clear()
        adapt._status_words.update(kept)


@pytest.mark.parametrize("T", [5, 40])
def test_an_input_in_a_graph_is_refused(T):
    from paper_2605_11222_b200 import adapt, binding as B
    g = _gen(43)
    codes, scale, zero = _layer(g, 128, 64, 4, 64)
    layer, bank, plan = adapt.QuantLinear(codes, scale, zero, 4, 64), _bank(g, 2, 8, 128, 64), _plan("mixed", T, 2)
    x = _randn(g, T, 128).bfloat16()
    want = layer.forward(x, bank, plan)
    out = torch.empty_like(want[0])
    leaf = x.clone().requires_grad_()
    for v in (leaf, leaf * 1):
        for call in (lambda: layer.forward(v), lambda: layer.forward(v, bank, plan), lambda: layer.forward(v, bank, plan, out=out)):
            with pytest.raises(adapt.AdmmqError, match="requires grad") as e:
                call()
            assert e.value.status == B.ERR_INVALID_ARG
        with torch.no_grad():
            assert torch.equal(layer.forward(v, bank, plan)[0], want[0])
    assert torch.equal(layer.forward(leaf.detach(), bank, plan)[0], want[0])
    with torch.inference_mode():
        assert torch.equal(layer.forward(x.clone(), bank, plan)[0], want[0])
    # adapters that require grad: as before
    bank = adapt.AdapterBank(bank.down.requires_grad_(), bank.up.requires_grad_(), bank.scale)
    assert torch.equal(layer.forward(x, bank, plan)[0], want[0])
    # a graph's node of its own
    class Layer(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x):
            return layer.forward(x, bank, plan)[0]

        @staticmethod
        def backward(ctx, dy):
            return layer.grad_input(dy, bank, plan)[0]

    y = Layer.apply(leaf)
    dy = _randn(g, T, 64).bfloat16()
    y.backward(dy)
    assert torch.equal(y, want[0]) and torch.equal(leaf.grad, layer.grad_input(dy, bank, plan)[0])
    # queries and keys
    q, w = _randn(g, T, 2, 64), torch.ones(64, device=DEV)
    cos, pos = torch.ones(T, 32, device=DEV), torch.arange(T, device=DEV, dtype=torch.int32)
    want = adapt.qk_norm_rope(q, q, w, w, cos, cos, pos)
    leaf = q.clone().requires_grad_()
    for a, b in ((leaf, q), (q, leaf)):
        with pytest.raises(adapt.AdmmqError, match="requires grad"):
            adapt.qk_norm_rope(a, b, w, w, cos, cos, pos)
        with torch.no_grad():
            assert all(torch.equal(s, t) for s, t in zip(adapt.qk_norm_rope(a, b, w, w, cos, cos, pos), want))
    adapt.qk_norm_rope(q, q, w.clone().requires_grad_(), w, cos, cos, pos)
    adapt.check_device_status(DEV)


# ------------------------------------------------------------------ checkpoints
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,n", [(0, 64), (1, 8), (3, 128), (5, 136), (77, 4096), (200, 1000), (2, 12288)])
def test_checkpoint_codes_scales_and_values(T, n, dtype):
    from paper_2605_11222_b200 import adapt
    g = _gen(T + n)
    big = _randn(g, T, n + 8) * 3
    if T > 1:
        big[0] = 0.0                              # a row of zeros
        big[1, ::3] *= 1e4
    x = big.to(dtype)[:, 8:]
    c = adapt.Checkpoint.save(x)
    nb = -(-n // 128)
    f = torch.zeros(T, nb * 128, device=DEV)
    f[:, :n] = x.float()
    f = f.view(T, nb, 128)
    scale = f.abs().amax(-1) / torch.full((), 127.0, device=DEV)
    codes = torch.where(scale[..., None] > 0, torch.round(f / scale[..., None]), torch.zeros_like(f))
    assert torch.equal(c.scale, scale)
    assert torch.equal(c.codes.float(), codes.view(T, nb * 128)[:, :n])
    want = (c.codes.float() * scale.repeat_interleave(128, 1)[:, :n]).to(dtype)
    assert torch.equal(c.restore(dtype), want)
    wide = torch.full((T, n + 8), 5.0, dtype=dtype, device=DEV)
    c.restore(dtype, out=wide[:, :n])
    assert torch.equal(wide[:, :n], want) and bool((wide[:, n:] == 5).all())
    # within half a step of what was kept
    assert bool(((c.restore(torch.float32) - x.float()).abs()
                 <= 0.5001 * scale.repeat_interleave(128, 1)[:, :n]).all())


def test_checkpoint_of_extreme_values():
    from paper_2605_11222_b200 import adapt
    x = torch.zeros(4, 256)
    x[0, 0], x[0, 1] = 3e38, -1.0
    x[1, 0], x[1, 1] = 1e-44, -1e-45              # subnormal: the scale is one of a few bits, or zero
    x[2, 5], x[2, 130] = float("nan"), 2.0
    x[3, 5], x[3, 130] = float("-inf"), 2.0
    r = adapt.Checkpoint.save(x.to(DEV)).restore(torch.float32).cpu()
    assert abs(r[0, 0] / 3e38 - 1) < 1e-6 and r[0, 1] == 0
    assert torch.isfinite(r[1]).all() and (r[1].abs() <= 1e-43).all()
    for t in (2, 3):
        assert torch.isnan(r[t, :128]).all()      # the block, and only it
        assert r[t, 130] == 2 and (r[t, 131:] == 0).all()


# ------------------------------------------------------------------ norm and rotation
def _qk64(x, w, cos, sin, rot, eps):
    n = x / (x.square().mean(-1, keepdim=True) + eps).sqrt()
    z = n * w
    a, b, rest = z[..., : rot // 2], z[..., rot // 2: rot], z[..., rot:]
    y = torch.cat([a * cos - b * sin, b * cos + a * sin, rest], -1)
    mag = torch.cat([a.abs() + b.abs(), a.abs() + b.abs(), rest.abs()], -1)
    return y, mag


QK = [(0, 4, 2, 64, 64), (1, 32, 8, 128, 128), (2, 1, 1, 16, 16), (3, 5, 0, 96, 32), (17, 12, 3, 64, 32), (33, 7, 7, 256, 256),
      (259, 3, 1, 80, 80), (1000, 6, 2, 128, 96), (5000, 4, 2, 48, 48), (9, 40, 33, 32, 16)]


def _qk_inputs(T, hq, hk, d, rot, dtype, g):
    big = (_randn(g, T, (hq + 2 * hk) * d + 16) * 2).to(dtype)
    q = big[:, : hq * d].view(T, hq, d) if T else torch.empty(0, hq, d, dtype=dtype, device=DEV)
    k = big[:, hq * d: (hq + hk) * d].view(T, hk, d) if T else torch.empty(0, hk, d, dtype=dtype, device=DEV)
    wq, wk = [(1 + 0.3 * _randn(g, d)).to(dtype) for _ in range(2)]
    ang = torch.arange(700, device=DEV)[:, None] * 1e4 ** (-torch.arange(0, rot, 2, device=DEV, dtype=torch.float64) / rot)
    pos = torch.randint(0, 700, (T,), generator=g, device=DEV, dtype=torch.int32)
    return q, k, wq, wk, ang.cos().float(), ang.sin().float(), pos


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,hq,hk,d,rot", QK)
def test_qk_norm_rope(T, hq, hk, d, rot, dtype):
    """fp32: the mean of squares over at most 256 values, its root, two products and the rotation, each a few half ulps:
    32 of them in all, of the magnitudes that enter the rotation; bf16 adds the output's rounding."""
    from paper_2605_11222_b200 import adapt
    g = _gen(T + d)
    q, k, wq, wk, cos, sin, pos = _qk_inputs(T, hq, hk, d, rot, dtype, g)
    yq, yk = adapt.qk_norm_rope(q, k, wq, wk, cos, sin, pos, 1e-6)
    adapt.check_device_status(DEV)
    c, s = cos.double()[pos.long()][:, None], sin.double()[pos.long()][:, None]
    half = EPS if dtype == torch.bfloat16 else 0.0
    for got, x, w in ((yq, q, wq), (yk, k, wk)):
        want, mag = _qk64(x.double(), w.double(), c, s, rot, 1e-6)
        _within(got, want, half * want.abs() + 32 * 2.0 ** -24 * mag + 1e-30)
    # in place
    q2, k2 = q.clone(), k.clone()
    adapt.qk_norm_rope(q2, k2, wq, wk, cos, sin, pos, 1e-6, out_q=q2, out_k=k2)
    assert torch.equal(q2, yq) and torch.equal(k2, yk)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,hq,hk,d,rot", QK)
def test_qk_norm_rope_backward(T, hq, hk, d, rot, dtype):
    """As forward, with r |dn| and r |n| mean |dn n| as the magnitudes that enter the last difference; weights: the
    sum's terms each with the same error, and the fp32 sum's own (64 half ulps of the sum of magnitudes)."""
    from paper_2605_11222_b200 import adapt
    g = _gen(T + d + 1)
    q, k, wq, wk, cos, sin, pos = _qk_inputs(T, hq, hk, d, rot, dtype, g)
    dyq, dyk = _randn(g, T, hq, d).to(dtype), _randn(g, T, hk, d).to(dtype)
    got = adapt.qk_norm_rope_backward(q, k, wq, wk, cos, sin, pos, dyq, dyk, 1e-6)
    adapt.check_device_status(DEV)
    c, s = cos.double()[pos.long()][:, None], sin.double()[pos.long()][:, None]
    half = EPS if dtype == torch.bfloat16 else 0.0
    h = rot // 2
    for gx, gw, x, w, dy in ((got[0], got[2], q, wq, dyq), (got[1], got[3], k, wk, dyk)):
        x, w, dy = x.double(), w.double(), dy.double()
        r = 1 / (x.square().mean(-1, keepdim=True) + 1e-6).sqrt()
        n = x * r
        a, b = dy[..., :h], dy[..., h:rot]
        gr = torch.cat([a * c + b * s, b * c - a * s, dy[..., rot:]], -1)
        ga = torch.cat([a.abs() + b.abs(), a.abs() + b.abs(), dy[..., rot:].abs()], -1)
        dn = gr * w
        want = r * (dn - n * (dn * n).mean(-1, keepdim=True))
        mag = r * (ga * w.abs() + n.abs() * (ga * w.abs() * n.abs()).mean(-1, keepdim=True))
        _within(gx, want, half * want.abs() + 64 * 2.0 ** -24 * mag + 1e-30)
        ww = (gr * n).sum((0, 1))
        _within(gw, ww, half * ww.abs() + 64 * 2.0 ** -24 * (ga * n.abs()).sum((0, 1)) + 1e-30)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,hq,hk,d,rot", [(1, 3, 2, 64, 32), (7, 1, 1, 128, 128), (260, 5, 2, 96, 64), (3000, 2, 3, 64, 64)])
def test_qk_strides_of_every_argument(T, hq, hk, d, rot, dtype):
    """Inputs, upstream gradients and outputs as views into joint buffers of different widths, heads apart and out of
    order: the bits of the dense call, and nothing written beside the views."""
    from paper_2605_11222_b200 import adapt
    g = _gen(T + 7)
    q, k, wq, wk, cos, sin, pos = _qk_inputs(T, hq, hk, d, rot, dtype, g)
    dyq, dyk = _randn(g, T, hq, d).to(dtype), _randn(g, T, hk, d).to(dtype)

    def views(a, b, pad):
        """a and b in one buffer: b's heads first, each head followed by `pad` other values, `pad` more at a row's end."""
        buf = torch.full((T, (hq + hk) * (d + pad) + pad), 9.0, dtype=dtype, device=DEV)
        vb = buf[:, :hk * (d + pad)].view(T, hk, d + pad)[..., :d]
        va = buf[:, hk * (d + pad):(hq + hk) * (d + pad)].view(T, hq, d + pad)[..., :d]
        if a is not None:
            va.copy_(a)
            vb.copy_(b)
        return va, vb, buf

    def untouched(va, vb, buf):
        va.fill_(9.0)
        vb.fill_(9.0)
        return bool((buf == 9).all())

    sq, sk, _ = views(q, k, 8)
    sdq, sdk, _ = views(dyq, dyk, 24)
    dense = adapt.qk_norm_rope(q.contiguous(), k.contiguous(), wq, wk, cos, sin, pos)
    assert all(torch.equal(a, b) for a, b in zip(adapt.qk_norm_rope(sq, sk, wq, wk, cos, sin, pos), dense))
    oq, ok, buf = views(None, None, 16)
    adapt.qk_norm_rope(sq, sk, wq, wk, cos, sin, pos, out_q=oq, out_k=ok)
    assert torch.equal(oq, dense[0]) and torch.equal(ok, dense[1]) and untouched(oq, ok, buf)
    dense = adapt.qk_norm_rope_backward(q.contiguous(), k.contiguous(), wq, wk, cos, sin, pos, dyq, dyk)
    got = adapt.qk_norm_rope_backward(sq, sk, wq, wk, cos, sin, pos, sdq, sdk)
    assert all(torch.equal(a, b) for a, b in zip(got, dense))
    got = adapt.qk_norm_rope_backward(sq, sk, wq, wk, cos, sin, pos, sdq, sdk, out_q=oq, out_k=ok)
    assert got[0] is oq and got[1] is ok
    assert all(torch.equal(a, b) for a, b in zip(got, dense)) and untouched(oq, ok, buf)
    adapt.check_device_status(DEV)


@pytest.mark.parametrize("T", [0, 1, 700])
def test_queries_without_keys(T):
    from paper_2605_11222_b200 import adapt
    g = _gen(T + 9)
    q, _, wq, wk, cos, sin, pos = _qk_inputs(T, 4, 0, 64, 64, torch.bfloat16, g)
    k = torch.empty(T, 0, 64, dtype=torch.bfloat16, device=DEV)
    dq = _randn(g, T, 4, 64).bfloat16()
    both, back = adapt.qk_norm_rope(q, q, wq, wq, cos, sin, pos), adapt.qk_norm_rope_backward(q, q, wq, wq, cos, sin, pos, dq, dq)
    yq, yk = adapt.qk_norm_rope(q, k, wq, wk, cos, sin, pos)
    assert torch.equal(yq, both[0]) and yk.shape == (T, 0, 64)
    gq, gk, gwq, gwk = adapt.qk_norm_rope_backward(q, k, wq, wk, cos, sin, pos, dq, torch.empty_like(k))
    assert torch.equal(gq, back[0]) and gk.shape == (T, 0, 64) and bool((gwk == 0).all())
    # another number of CTAs adds the weight's gradient in another order: two roundings of the output, and 64 half ulps of
    # the sum of magnitudes (4 T terms of less than 2.5 on average) in each
    assert bool(((gwq.float() - back[2].float()).abs() <= 2 * EPS * back[2].float().abs() + 2.0 ** -17 * 10 * T).all())
    adapt.check_device_status(DEV)


def test_qk_gradient_agrees_with_differences():
    """Central differences of the fp32 forward call: error of order step^2 third derivatives plus the forward's
    rounding over the step; both are below 1e-3 of the gradient's scale at the step used."""
    from paper_2605_11222_b200 import adapt
    g = _gen(4)
    T, hq, hk, d, rot = 6, 3, 2, 64, 32
    q, k, wq, wk, cos, sin, pos = [t.contiguous() for t in _qk_inputs(T, hq, hk, d, rot, torch.float32, g)]
    cq, ck = _randn(g, T, hq, d), _randn(g, T, hk, d)
    grads = adapt.qk_norm_rope_backward(q, k, wq, wk, cos, sin, pos, cq, ck, 1e-6)

    def loss(v):
        a, b = adapt.qk_norm_rope(*v, cos, sin, pos, 1e-6)
        return float((a.double() * cq.double()).sum() + (b.double() * ck.double()).sum())

    for i in range(4):
        v = [q, k, wq, wk]
        step = _randn(g, *v[i].shape)
        e = 2e-3
        hi, lo = list(v), list(v)
        hi[i], lo[i] = v[i] + e * step, v[i] - e * step
        got = (loss(hi) - loss(lo)) / (2 * e)
        want = float((grads[i].double() * step.double()).sum())
        size = float((grads[i].double() * step.double()).square().sum().sqrt()) + 1.0
        assert abs(got - want) <= 1e-2 * size, (i, got, want)


def test_qk_refusals_and_positions_out_of_range():
    from paper_2605_11222_b200 import adapt, binding as B
    g = _gen(7)
    q, k, wq, wk, cos, sin, pos = _qk_inputs(4, 2, 1, 64, 64, torch.float32, g)

    def refused(status, *a, **kw):
        with pytest.raises(adapt.AdmmqError) as e:
            adapt.qk_norm_rope(*a, **kw)
        assert e.value.status == status

    refused(B.ERR_INVALID_ARG, q.half(), k.half(), wq, wk, cos, sin, pos)
    refused(B.ERR_INVALID_ARG, q, k, wq.bfloat16(), wk, cos, sin, pos)
    refused(B.ERR_SHAPE, q, k, wq, wk, cos[:, :12].contiguous(), sin[:, :12].contiguous(), pos)
    refused(B.ERR_INVALID_ARG, q, k, wq, wk, cos, sin, pos.long())
    refused(B.ERR_SHAPE, q[..., :40], k[..., :40], wq[:40], wk[:40], cos[:, :16].contiguous(), sin[:, :16].contiguous(), pos)
    refused(B.ERR_INVALID_ARG, q, k, wq, wk, cos, sin, pos, -1.0)
    pos[2] = 700
    adapt.qk_norm_rope(q, k, wq, wk, cos, sin, pos)
    with pytest.raises(adapt.AdmmqError) as e:
        adapt.check_device_status(DEV)
    assert e.value.status == B.ERR_SHAPE
    adapt.check_device_status(DEV)


def test_the_example_trains_its_adapters():
    """The operators together, as the example uses them: the loss falls (the gradients point the right way through the
    rotation, the norm, the codes and the 8-bit inputs), and a request without an adapter gets the bare layer."""
    import os
    import sys
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import adapt_attention_input as ex
    losses, dx, same = ex.main(hidden=512, steps=12, rank=8, rows=200, quiet=True)
    assert losses[-1] < 0.9 * losses[0] and all(math.isfinite(v) for v in losses)
    assert dx.shape == (200, 512) and torch.isfinite(dx.float()).all()
    assert same

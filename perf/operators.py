"""Cases that measure the operators on quantised layers: the shared projection with the adapters of many requests
(serving, and the backward pass of training adapters), 8-bit activation checkpoints, and the per-head norm of queries
and keys with the position rotation (forward and backward).

Layer sizes are those of the 36-block stack of the solver's benchmark (hidden 4096, MLP 12288, KV width 1024), with
its grids: W3 and W4 asymmetric with groups of 128, W2 symmetric per output channel; and odd ones between.

`own` false: the operators in elementary torch operations in 32 bits.  `own` true: this repository's calls.
"""
import math

import torch

own = False

BLOCK = 128            # channels that share one scale of an 8-bit checkpoint
EPS = 1e-6
HEAD_TABLE = 40960     # positions in the rotation table


# ------------------------------------------------------------------ cases
def listed():
    return [
        # one new token of one request through q_proj: the latency of decoding
        dict(name="linear_one_token", op="linear", tokens=1, d_in=4096, d_out=4096, bits=4, group=128, sym=False,
             adapters=8, rank=16, requests=1, phase="decode"),
        # a decoding batch, each request with an adapter of its own or none, through k_proj as W2 per channel
        dict(name="linear_decode_batch", op="linear", tokens=13, d_in=4096, d_out=1024, bits=2, group=0, sym=True,
             adapters=16, rank=8, requests=13, phase="decode"),
        # a step that mixes decoding requests and pieces of prompts, through gate_proj
        dict(name="linear_mixed_step", op="linear", tokens=203, d_in=4096, d_out=12288, bits=4, group=128, sym=False,
             adapters=24, rank=32, requests=31, phase="mixed"),
        # prompts of several requests, ragged, through q_proj as W3
        dict(name="linear_prefill", op="linear", tokens=6011, d_in=4096, d_out=4096, bits=3, group=128, sym=False,
             adapters=4, rank=16, requests=7, phase="mixed"),
        # backward of a short training batch of a KV projection: rank 64, three adapters of which one may stay unused
        dict(name="backward_short", op="backward", tokens=333, d_in=4096, d_out=1024, bits=4, group=128, sym=False,
             adapters=3, rank=64, requests=3, phase="mixed"),
        # backward of a full training batch of down_proj, one adapter
        dict(name="backward_long", op="backward", tokens=8192, d_in=12288, d_out=4096, bits=4, group=128, sym=False,
             adapters=1, rank=16, requests=1, phase="mixed"),
        # activations of a few sequences kept in 8 bits and restored
        dict(name="checkpoint_short", op="checkpoint", tokens=77, width=4096, dtype="bf16"),
        # the input of down_proj for a full batch
        dict(name="checkpoint_long", op="checkpoint", tokens=16384, width=12288, dtype="bf16"),
        # one new token: 32 query and 8 key heads of 128
        dict(name="qk_one_token", op="qk", tokens=1, q_heads=32, k_heads=8, head=128, rot=128, dtype="bf16",
             backward=False),
        # prompts: q and k taken out of one joint buffer
        dict(name="qk_prefill", op="qk", tokens=16384, q_heads=32, k_heads=8, head=128, rot=128, dtype="bf16",
             backward=False),
        # gradient in 32 bits, small heads of which a half is rotated
        dict(name="qk_backward_short", op="qk", tokens=259, q_heads=12, k_heads=3, head=64, rot=32, dtype="f32",
             backward=True),
        # gradient of a full batch
        dict(name="qk_backward_long", op="qk", tokens=8192, q_heads=32, k_heads=8, head=128, rot=128, dtype="bf16",
             backward=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo):
    """A width that no configuration has: an odd multiple of 8, from about 8 lo up to 5128 channels."""
    return 8 * (2 * rng.randint(lo // 2, 320) + 1)


def _grid(rng, d_in):
    bits = rng.choice([2, 3, 4])
    group = rng.choice([0, 64, 128, 256])
    return bits, (group if group and d_in % group == 0 else 0), rng.random() < 0.3


def draw(rng):
    op = rng.choice(["linear", "linear", "backward", "checkpoint", "qk"])
    if op == "linear" or op == "backward":
        d_in = rng.choice([4096, 4096, 12288, _width(rng, 32)])
        d_out = rng.choice([1024, 4096, 4096, 12288, _width(rng, 16)])
        if op == "linear":
            phase = rng.choice(["decode", "mixed"])
            tokens = _log_int(rng, 1, 64) if phase == "decode" else _log_int(rng, 17, 6000)
        else:
            phase, tokens = "mixed", _log_int(rng, 64, 8000)
        tokens = max(1, min(tokens, 6000 * 4096 * 4096 // (d_in * d_out)))
        bits, group, sym = _grid(rng, d_in)
        requests = tokens if phase == "decode" else min(tokens, _log_int(rng, 1, 40))
        return dict(op=op, tokens=tokens, d_in=d_in, d_out=d_out, bits=bits, group=group, sym=sym,
                    adapters=_log_int(rng, 1, 24), rank=rng.choice([8, 16, 24, 32, 64]), requests=requests,
                    phase=phase)
    if op == "checkpoint":
        return dict(op=op, tokens=_log_int(rng, 1, 16000), width=rng.choice([4096, 12288, _width(rng, 16)]),
                    dtype=rng.choice(["bf16", "bf16", "f32"]))
    head = rng.choice([64, 96, 128, 128, 256])
    k_heads = rng.randint(1, 8)
    backward = rng.random() < 0.5
    q_heads = k_heads * rng.randint(1, 4)
    return dict(op=op, tokens=_log_int(rng, 1, 8000), q_heads=q_heads, k_heads=k_heads, head=head,
                rot=rng.choice([head, head, 32]), dtype=rng.choice(["bf16", "bf16", "f32"]), backward=backward)


# ------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _activations(g, rows, width):
    """N(0, 1) channels, one in a hundred of them large and heavy-tailed (Student-t of 3 degrees, times 30)."""
    x = torch.randn(rows, width, generator=g, device="cuda")
    m = max(1, width // 100)
    ch = torch.randperm(width, generator=g, device="cuda")[:m]
    z = torch.randn(rows, m, 4, generator=g, device="cuda")
    x[:, ch] = 30.0 * z[..., 0] / torch.sqrt((z[..., 1:] ** 2).sum(-1) / 3.0)
    return x


def _quantised(g, c):
    """Codes and grid of a layer N(0, 0.02^2): the min-max grid of every group, rounded to nearest."""
    p, n = c["d_out"], c["d_in"]
    gs = c["group"] or n
    w = (torch.randn(p, n, generator=g, device="cuda") * 0.02).view(p, n // gs, gs)
    lo, hi = w.amin(-1), w.amax(-1)
    if c["sym"]:
        hi = torch.maximum(hi, -lo)
        lo = -hi
    top = 2 ** c["bits"] - 1
    scale = (hi - lo) / top
    codes = torch.round((w - lo[..., None]) / scale[..., None]).clamp_(0, top).to(torch.uint8).view(p, n)
    return codes, scale, lo


def _requests(seed, c):
    """Lengths of the requests (ragged, their sum is the number of tokens) and the adapter of each (-1: none)."""
    g = torch.Generator()
    g.manual_seed(seed * 31 + 7)
    n, t = c["requests"], c["tokens"]
    if c["phase"] == "decode":
        lengths = [1] * n
    else:
        cuts = torch.randint(0, t + 1, (n - 1,), generator=g).sort().values.tolist()
        lengths = [b - a for a, b in zip([0] + cuts, cuts + [t])]
    low = 0 if c["adapters"] == 1 else -1
    adapters = torch.randint(low, c["adapters"], (n,), generator=g).tolist()
    return lengths, adapters


def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _save_plain(x):
    """8-bit checkpoint of x [T, n]: codes int8, one scale for every row and block of channels."""
    t, n = x.shape
    nb = -(-n // BLOCK)
    f = torch.zeros(t, nb * BLOCK, device=x.device)
    f[:, :n] = x.float()
    f = f.view(t, nb, BLOCK)
    scale = f.abs().amax(-1) / 127.0
    safe = torch.where(scale > 0, scale, torch.ones_like(scale))
    codes = torch.round(f / safe[..., None]).clamp(-127, 127).to(torch.int8).view(t, nb * BLOCK)[:, :n]
    return codes.contiguous(), scale


def _restore_plain(codes, scale):
    return codes.float() * scale.repeat_interleave(BLOCK, 1)[:, : codes.shape[1]]


def prepare(case, seed):
    c = dict(case)
    g = _gen(seed)
    s = {"case": c}
    if c["op"] in ("linear", "backward"):
        t, n, p, r, na = c["tokens"], c["d_in"], c["d_out"], c["rank"], c["adapters"]
        s["codes"], s["scale"], s["zero"] = _quantised(g, c)
        # trained adapters: down as initialised (uniform, 1 / sqrt(n) wide), up a few training steps away from zero
        s["down"] = ((torch.rand(na, r, n, generator=g, device="cuda") * 2 - 1) / math.sqrt(n)).bfloat16()
        s["up"] = (torch.randn(na, r, p, generator=g, device="cuda") * 0.02).bfloat16()
        s["alpha"] = torch.full((na,), 2.0, device="cuda") / (1 + torch.arange(na, device="cuda") % 3)
        lengths, adapters = _requests(seed, c)
        s["row_adapter"] = torch.repeat_interleave(torch.tensor(adapters), torch.tensor(lengths)).cuda()
        x = _activations(g, t, n).bfloat16()
        if c["op"] == "linear":
            s["x"] = x
        else:
            s["x_codes"], s["x_scale"] = _save_plain(x)
            s["dy"] = (torch.randn(t, p, generator=g, device="cuda") * 1e-3).bfloat16()
            s["h"] = _shrink(x, s["down"], s["row_adapter"], s["alpha"])
        if own:
            from paper_2605_11222_b200 import adapt
            s["layer"] = adapt.QuantLinear(s["codes"], s["scale"], s["zero"], c["bits"], c["group"])
            s["bank"] = adapt.AdapterBank(s["down"], s["up"], s["alpha"])
            s["plan"] = adapt.RequestPlan(lengths, adapters, na)
            if c["op"] == "backward":
                s["checkpoint"] = adapt.Checkpoint(s["x_codes"], s["x_scale"])
    elif c["op"] == "checkpoint":
        s["x"] = _activations(g, c["tokens"], c["width"]).to(_dtype(c))
    else:
        t, hq, hk, d, rot = c["tokens"], c["q_heads"], c["k_heads"], c["head"], c["rot"]
        # queries, keys and values side by side in one buffer, as a joint projection leaves them
        qkv = (torch.randn(t, (hq + 2 * hk) * d, generator=g, device="cuda") * 1.5).to(_dtype(c))
        s["q"] = qkv[:, : hq * d].view(t, hq, d)
        s["k"] = qkv[:, hq * d: (hq + hk) * d].view(t, hk, d)
        s["wq"] = (1 + 0.2 * torch.randn(d, generator=g, device="cuda")).to(_dtype(c))
        s["wk"] = (1 + 0.2 * torch.randn(d, generator=g, device="cuda")).to(_dtype(c))
        inv = 1e6 ** (-torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / rot)
        ang = torch.arange(HEAD_TABLE, device="cuda", dtype=torch.float64)[:, None] * inv
        s["cos"], s["sin"] = ang.cos().float(), ang.sin().float()
        first = int(torch.randint(0, HEAD_TABLE - t, (1,), generator=g, device="cuda"))
        s["pos"] = torch.arange(first, first + t, device="cuda", dtype=torch.int32)
        if c["backward"]:
            s["dq"] = torch.randn(t, hq, d, generator=g, device="cuda").to(_dtype(c))
            s["dk"] = torch.randn(t, hk, d, generator=g, device="cuda").to(_dtype(c))
    return s


# ------------------------------------------------------------------ plain forms, 32 bits
def _weight(s):
    p, n = s["codes"].shape
    groups = s["scale"].shape[1]
    k = s["codes"].view(p, groups, n // groups).float()
    return (s["zero"][..., None] + s["scale"][..., None] * k).view(p, n)


def _chosen(row_adapter, alpha):
    """[T, adapters]: the scale of the row's adapter at its place, zero elsewhere."""
    return (row_adapter[:, None] == torch.arange(alpha.numel(), device=alpha.device)) * alpha


def _own_rank(all_h, row_adapter):
    """[T, adapters, r] -> [T, r]: the row's own adapter's values (zero without one)."""
    at = row_adapter.clamp(min=0)[:, None, None].expand(-1, 1, all_h.shape[2])
    return all_h.gather(1, at)[:, 0] * (row_adapter >= 0)[:, None]


def _shrink(x, mat, row_adapter, alpha):
    """s_a mat_a x_t for every row: through all adapters at once, the row's own one kept."""
    na, r, n = mat.shape
    every = (x.float() @ mat.float().view(na * r, n).T).view(-1, na, r)
    return _own_rank(every * _chosen(row_adapter, alpha)[..., None], row_adapter)


def _expand(u, mat, row_adapter):
    """mat_a^T u_t for every row."""
    na, r, n = mat.shape
    one = (row_adapter[:, None] == torch.arange(na, device=u.device)).float()
    return (one[..., None] * u[:, None]).view(-1, na * r) @ mat.float().view(na * r, n)


def _outer(u, v, row_adapter, na):
    """sum over an adapter's rows of u_t v_t^T: [adapters, r, n]."""
    one = (row_adapter[:, None] == torch.arange(na, device=u.device)).float()
    return ((one[..., None] * u[:, None]).view(u.shape[0], -1).T @ v).view(na, u.shape[1], v.shape[1])


def _halves(x, rot):
    return x[..., : rot // 2], x[..., rot // 2: rot], x[..., rot:]


def _turn(x, cos, sin, rot):
    a, b, rest = _halves(x, rot)
    return torch.cat([a * cos - b * sin, b * cos + a * sin, rest], -1)


def _qk_plain(x, w, cos, sin, rot):
    x = x.float()
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    return _turn(x * r * w.float(), cos, sin, rot)


def _qk_plain_backward(x, w, dy, cos, sin, rot):
    x = x.float()
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    n = x * r
    g = _turn(dy.float(), cos, -sin, rot)
    dn = g * w.float()
    return r * (dn - n * (dn * n).mean(-1, keepdim=True)), (g * n).sum((0, 1))


def _run_plain(s):
    c = s["case"]
    if c["op"] == "linear":
        h = _shrink(s["x"], s["down"], s["row_adapter"], s["alpha"])
        y = s["x"].float() @ _weight(s).T + _expand(h, s["up"], s["row_adapter"])
        return y.bfloat16()
    if c["op"] == "backward":
        dy = s["dy"].float()
        u = _shrink(dy, s["up"], s["row_adapter"], s["alpha"])
        dx = dy @ _weight(s) + _expand(u, s["down"], s["row_adapter"])
        x = _restore_plain(s["x_codes"], s["x_scale"])
        d_down = _outer(u, x, s["row_adapter"], c["adapters"])
        d_up = _outer(s["h"], dy, s["row_adapter"], c["adapters"])
        return dx.bfloat16(), d_down.bfloat16(), d_up.bfloat16()
    if c["op"] == "checkpoint":
        codes, scale = _save_plain(s["x"])
        return _restore_plain(codes, scale).to(s["x"].dtype)
    cos, sin = s["cos"][s["pos"].long()][:, None], s["sin"][s["pos"].long()][:, None]
    t = s["q"].dtype
    if not c["backward"]:
        return (_qk_plain(s["q"], s["wq"], cos, sin, c["rot"]).to(t),
                _qk_plain(s["k"], s["wk"], cos, sin, c["rot"]).to(t))
    dq, dwq = _qk_plain_backward(s["q"], s["wq"], s["dq"], cos, sin, c["rot"])
    dk, dwk = _qk_plain_backward(s["k"], s["wk"], s["dk"], cos, sin, c["rot"])
    return dq.to(t), dk.to(t), dwq.to(t), dwk.to(t)


def run(state):
    s = state
    if not own:
        return _run_plain(s)
    from paper_2605_11222_b200 import adapt
    op = s["case"]["op"]
    if op == "linear":
        return s["layer"].forward(s["x"], s["bank"], s["plan"])[0]
    if op == "backward":
        dx, u = s["layer"].grad_input(s["dy"], s["bank"], s["plan"])
        d_down, d_up = adapt.adapter_grads(s["bank"], s["plan"], s["checkpoint"], s["h"], s["dy"], u)
        return dx, d_down, d_up
    if op == "checkpoint":
        return adapt.Checkpoint.save(s["x"]).restore(s["x"].dtype)
    if not s["case"]["backward"]:
        return adapt.qk_norm_rope(s["q"], s["k"], s["wq"], s["wk"], s["cos"], s["sin"], s["pos"], EPS)
    return adapt.qk_norm_rope_backward(s["q"], s["k"], s["wq"], s["wk"], s["cos"], s["sin"], s["pos"],
                                       s["dq"], s["dk"], EPS)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    c = case
    if c["op"] in ("linear", "backward"):
        t, n, p, r = c["tokens"], c["d_in"], c["d_out"], c["rank"]
        groups = n // (c["group"] or n)
        used = min(c["adapters"], c["requests"])
        layer = p * n * c["bits"] / 8 + 8 * p * groups + used * 2 * r * (n + p)
        if c["op"] == "linear":
            return {"bytes": layer + 2 * t * (n + p), "flops": 2 * t * n * p + 2 * t * r * (n + p)}
        kept = t * n + 4 * t * -(-n // BLOCK) + 4 * t * r
        return {"bytes": layer + kept + 2 * t * (n + p) + c["adapters"] * 2 * r * (n + p),
                "flops": 2 * t * n * p + 4 * t * r * (n + p)}
    if c["op"] == "checkpoint":
        e = 2 if c["dtype"] == "bf16" else 4
        t, n = c["tokens"], c["width"]
        return {"bytes": t * n * (2 * e + 1) + 4 * t * -(-n // BLOCK), "flops": 3 * t * n}
    e = 2 if c["dtype"] == "bf16" else 4
    t, h, d = c["tokens"], c["q_heads"] + c["k_heads"], c["head"]
    table = 4 * t * c["rot"] + 4 * t
    if c["backward"]:
        return {"bytes": 3 * e * t * h * d + 4 * e * d + table, "flops": 14 * t * h * d}
    return {"bytes": 2 * e * t * h * d + 2 * e * d + table, "flops": 8 * t * h * d}


# ------------------------------------------------------------------ the definitions in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    c = s["case"]
    f64 = torch.float64
    if c["op"] in ("linear", "backward"):
        n = c["d_in"]
        at = torch.arange(n, device="cuda") // (c["group"] or n)
        w = s["zero"].to(f64)[:, at] + s["scale"].to(f64)[:, at] * s["codes"].to(f64)
        down, up, alpha = s["down"].to(f64), s["up"].to(f64), s["alpha"].to(f64)
        rows = [(s["row_adapter"] == a).nonzero()[:, 0] for a in range(c["adapters"])]
        if c["op"] == "linear":
            x = s["x"].to(f64)
            y = torch.einsum("ti,ji->tj", x, w)
            for a, t in enumerate(rows):
                y[t] += alpha[a] * torch.einsum("ti,ri,rj->tj", x[t], down[a], up[a])
            return y
        dy, h = s["dy"].to(f64), s["h"].to(f64)
        at = torch.arange(n, device="cuda") // BLOCK
        x = s["x_codes"].to(f64) * s["x_scale"].to(f64)[:, at]
        dx = torch.einsum("tj,ji->ti", dy, w)
        d_down, d_up = torch.zeros_like(down), torch.zeros_like(up)
        for a, t in enumerate(rows):
            u = alpha[a] * torch.einsum("tj,rj->tr", dy[t], up[a])
            dx[t] += torch.einsum("tr,ri->ti", u, down[a])
            d_down[a] = torch.einsum("tr,ti->ri", u, x[t])
            d_up[a] = torch.einsum("tr,tj->rj", h[t], dy[t])
        return dx, d_down, d_up
    if c["op"] == "checkpoint":
        # the stored scale has 32 bits and the code is the nearest whole number of them: part of the definition
        x = s["x"].to(f64)
        out = torch.empty_like(x)
        for b in range(0, c["width"], BLOCK):
            part = x[:, b: b + BLOCK]
            scale = (part.abs().amax(1, keepdim=True).float() / 127.0).to(f64)
            k = torch.where(scale > 0, torch.round((part / scale).float().to(f64)), torch.zeros_like(part))
            out[:, b: b + BLOCK] = k * scale
        return out
    cos, sin = s["cos"].to(f64)[s["pos"].long()], s["sin"].to(f64)[s["pos"].long()]
    half, rot = c["rot"] // 2, c["rot"]
    # the rotation as one matrix for every position, its transpose in the gradient
    turn = torch.eye(c["head"], device="cuda", dtype=f64).repeat(c["tokens"], 1, 1)
    i = torch.arange(half, device="cuda")
    turn[:, i, i], turn[:, i + half, i + half] = cos, cos
    turn[:, i, i + half], turn[:, i + half, i] = -sin, sin
    out, grads = [], []
    for x, w, dy in ((s["q"], s["wq"], s.get("dq")), (s["k"], s["wk"], s.get("dk"))):
        x, w = x.to(f64), w.to(f64)
        ms = x.square().mean(-1, keepdim=True) + EPS
        if dy is None:
            out.append(torch.einsum("tij,thj->thi", turn, w * x / ms.sqrt()))
            continue
        g = torch.einsum("tji,thj->thi", turn, dy.to(f64))
        out.append(g * w / ms.sqrt() - x * (g * w * x).sum(-1, keepdim=True) / (c["head"] * ms ** 1.5))
        grads.append((g * x / ms.sqrt()).sum((0, 1)))
    return tuple(out + grads)

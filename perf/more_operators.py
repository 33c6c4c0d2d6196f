"""Cases that measure the cache of keys and values in 8 bits: writing rows into it as they come and reading them back,
attention of new tokens (one, a few, prompts) over it, and a decoding step of both.

Heads are those of the 36-block stack of the solver's benchmark (32 query and 8 key heads of 128) and of the example
(64 wide), and odd ones between.  A block of 16 tokens of one head shares a scale; pages hold 16 to 256 tokens.

`own` false: the operators in elementary torch operations in 32 bits.  `own` true: this repository's calls.
"""
import math
import random

import torch

own = False

BLOCK = 16             # tokens that share the scale of a head


# ------------------------------------------------------------------ cases
def listed():
    return [
        # one new token of one request: the latency of decoding
        dict(name="attend_one_token", op="attend", requests=1, new=1, prompt=0, held=1000, q_heads=32, k_heads=8,
             head=128, page=64, window=0),
        # a decoding batch of ragged requests
        dict(name="attend_batch", op="attend", requests=48, new=1, prompt=0, held=6000, q_heads=32, k_heads=8, head=128,
             page=64, window=0),
        # two requests far into long documents: few heads to share the work out over
        dict(name="attend_long", op="attend", requests=2, new=1, prompt=0, held=100_001, q_heads=32, k_heads=8, head=128,
             page=128, window=0),
        # three drafted tokens of each request to be verified, narrow heads, within a window
        dict(name="attend_drafts", op="attend", requests=7, new=3, prompt=0, held=2500, q_heads=15, k_heads=3, head=64,
             page=16, window=1000),
        # a step that mixes decoding requests and a piece of a prompt
        dict(name="attend_mixed", op="attend", requests=24, new=1, prompt=700, held=3000, q_heads=32, k_heads=8,
             head=128, page=32, window=0),
        # the next piece of a long document
        dict(name="attend_piece", op="attend", requests=1, new=512, prompt=0, held=32_768, q_heads=32, k_heads=8,
             head=128, page=64, window=0),
        # a whole prompt
        dict(name="attend_prompt", op="attend", requests=1, new=8192, prompt=0, held=0, q_heads=32, k_heads=8, head=128,
             page=64, window=0),
        # one new token written behind those of its block, and the block read back
        dict(name="store_one_token", op="store", requests=1, new=1, prompt=0, held=1003, k_heads=8, head=128, page=64,
             dtype="bf16"),
        # a token of every request of a batch, fp32, odd heads
        dict(name="store_batch", op="store", requests=77, new=1, prompt=0, held=900, k_heads=5, head=96, page=32,
             dtype="f32"),
        # prompts of several requests, and all of them read back (a cache handed on)
        dict(name="store_prompts", op="store", requests=6, new=5000, prompt=0, held=0, k_heads=8, head=128, page=64,
             dtype="bf16"),
        # a decoding step: the new tokens written, then attended with
        dict(name="step_one_token", op="step", requests=1, new=1, prompt=0, held=4100, q_heads=32, k_heads=8, head=128,
             page=64, window=0),
        dict(name="step_batch", op="step", requests=128, new=1, prompt=0, held=9000, q_heads=32, k_heads=8, head=128,
             page=64, window=0),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["attend", "attend", "attend", "store", "step"])
    k_heads, page = rng.randint(1, 8), rng.choice([16, 32, 64, 128, 256])
    head = rng.choice([64, 96, 128, 128, 256])
    if op == "store":
        requests = _log_int(rng, 1, 80)
        new = 1 if rng.random() < 0.5 else _log_int(rng, 2, 5000)
        return dict(op=op, requests=requests if new == 1 else min(requests, 6), new=new, prompt=0,
                    held=_log_int(rng, 1, 4000), k_heads=k_heads, head=head, page=page, dtype=rng.choice(["bf16", "f32"]))
    q_heads = k_heads * rng.choice([1, 2, 3, 4, 5, 7, 8])
    q_heads = min(q_heads, 32 // k_heads * k_heads)
    kind = "tokens" if op == "step" else rng.choice(["tokens", "tokens", "drafts", "mixed", "prompts"])
    requests, new, prompt, held = 1, 1, 0, 0
    if kind == "tokens":
        requests = _log_int(rng, 1, 100)
        held = _log_int(rng, 1, min(100_000, 600_000 // requests, 600_000_000 // (requests * k_heads * head)))
    elif kind == "drafts":
        requests, new, held = _log_int(rng, 1, 40), rng.randint(2, 9), _log_int(rng, 1, 6000)
    elif kind == "mixed":
        requests, prompt, held = _log_int(rng, 1, 24), _log_int(rng, 20, 700), _log_int(rng, 1, 3000)
    else:
        requests, new = rng.randint(1, 3), _log_int(rng, 30, 4000)
        held = _log_int(rng, 1, 4000)
    return dict(op=op, requests=requests, new=new, prompt=prompt, held=held, q_heads=q_heads, k_heads=k_heads, head=head,
                page=page, window=rng.choice([0, 0, _log_int(rng, 1, 4000)]))


def _lengths(c):
    """(new tokens, tokens held before them) of every request: ragged, the first ones the longest."""
    rng = random.Random(repr(sorted((k, v) for k, v in c.items() if k != "name")))
    new, held = [], []
    for i in range(c["requests"]):
        new.append(c["new"] if i == 0 or c["new"] < 10 else rng.randint(c["new"] // 4, c["new"]))
        held.append(c["held"] if i == 0 else rng.randint(c["held"] // 4, c["held"]))
    if c["prompt"]:
        new.append(c["prompt"])
        held.append(rng.randint(0, c["held"]))
    return new, held


# ------------------------------------------------------------------ inputs
def _dtype(c):
    return torch.float32 if c.get("dtype") == "f32" else torch.bfloat16


def _rows(g, t, heads, d, dtype):
    """Keys or values: N(0, 1), one channel in fifty five times as large."""
    x = torch.randn(t, heads, d, generator=g, device="cuda")
    wide = torch.randperm(d, generator=g, device="cuda")[: max(1, d // 50)]
    x[..., wide] *= 5.0
    return x.to(dtype)


def _units(new, first, tables, page):
    """The blocks that a plan's rows touch: place in the pool (page, block of the page), first row, first slot, rows."""
    out, row = [], 0
    for i, (n, p) in enumerate(zip(new, first)):
        end, at = p + n, p
        while at < end:
            stop = min(end, at - at % BLOCK + BLOCK)
            out.append((tables[i][at // page], at % page // BLOCK, row + at - p, at % BLOCK, stop - at))
            at = stop
        row += n
    return torch.tensor(out, dtype=torch.int64).view(-1, 5).cuda()


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    new, held = _lengths(c)
    page, hk, d = c["page"], c["k_heads"], c["head"]
    need = [-(-(n + p) // page) for n, p in zip(new, held)]
    n_pages = sum(need) + 3
    order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed)).tolist()
    tables = [order[sum(need[:i]): sum(need[: i + 1])] for i in range(len(need))]
    wide = max(need)
    padded = torch.tensor([t + [0] * (wide - len(t)) for t in tables], dtype=torch.int32).cuda()
    s = {"case": c, "tables": padded, "held": torch.tensor(held, dtype=torch.int32).cuda(),
         "new": torch.tensor(new, dtype=torch.int32).cuda()}
    # what the cache holds before the pass: the earlier tokens, and where only attention is measured the new ones too
    filled = [n + p for n, p in zip(new, held)] if c["op"] == "attend" else held
    fk, fv = _rows(g, sum(filled), hk, d, torch.bfloat16), _rows(g, sum(filled), hk, d, torch.bfloat16)
    nothing = [0] * len(new)
    starts = [0] + torch.tensor(new).cumsum(0).tolist()
    s["first_row"] = torch.tensor(starts[:-1]).cuda()
    s["units"] = _units(new, held, tables, page)
    # the rows of a pass: keys and values side by side in one buffer, as a joint projection leaves them
    kv = _rows(g, sum(new), 2 * hk, d, _dtype(c))
    s["k"], s["v"] = kv[:, :hk], kv[:, hk:]
    if c["op"] != "store":
        s["q"] = (1.5 * torch.randn(sum(new), c["q_heads"], d, generator=g, device="cuda")).bfloat16()
        s["row_request"] = torch.repeat_interleave(torch.arange(len(new)), torch.tensor(new)).cuda()
        s["row_index"] = torch.cat([torch.arange(n) for n in new]).cuda()
    # the tokens read back: those of every block that is written to
    begin = [p - p % BLOCK for p in held]
    seen = [p + n - b for p, n, b in zip(held, new, begin)]
    s["seen_at"] = _positions(begin, seen, tables, page)
    if own:
        from paper_2605_11222_b200 import kvcache
        s["cache"] = kvcache.KVCache(n_pages, hk, d, page)
        s["cache"].write(fk, fv, kvcache.CachePlan(filled, nothing, padded))
        s["plan"] = kvcache.CachePlan(new, s["held"], padded, group=c.get("q_heads", hk) // hk)
        s["seen"] = kvcache.CachePlan(seen, begin, padded)
    else:
        # per page: the codes of every head and token, and a scale a block
        s["codes"] = [torch.zeros(n_pages, hk, page, d, dtype=torch.int8, device="cuda") for _ in "kv"]
        s["scale"] = [torch.zeros(n_pages, hk, page // BLOCK, device="cuda") for _ in "kv"]
        at = _units(filled, nothing, tables, page)
        _write_plain(s["codes"][0], s["scale"][0], fk, at)
        _write_plain(s["codes"][1], s["scale"][1], fv, at)
    return s


def _positions(begin, count, tables, page):
    """(page, slot of the page) of the tokens begin .. begin + count of every request."""
    out = [(tables[i][p // page], p % page) for i, (b, n) in enumerate(zip(begin, count)) for p in range(b, b + n)]
    return torch.tensor(out, dtype=torch.int64).view(-1, 2).cuda()


# ------------------------------------------------------------------ plain forms, 32 bits
def _write_plain(codes, scale, x, units):
    """Rows x [T, heads, D] into the blocks of `units`.  A block's scale is the largest magnitude that it was given,
    over 127; where it grows, the codes that the block holds are rounded to the new one."""
    if units.shape[0] == 0:
        return
    pages, blk, row, slot, n = units.unbind(1)
    h, d = codes.shape[1], codes.shape[3]
    at = torch.arange(BLOCK, device=x.device)[None] - slot[:, None]                    # row of the unit, by slot
    fresh = ((at >= 0) & (at < n[:, None]))[:, None, :, None]                          # [units, 1, 16, 1]
    rows = (row[:, None] + at).clamp(0, x.shape[0] - 1)
    v = x[rows].float().transpose(1, 2) * fresh                                        # [units, heads, 16, D]
    old = scale[pages, :, blk] * (slot > 0)[:, None]
    grid = codes.view(codes.shape[0], h, -1, BLOCK, d)
    now = torch.maximum(old, v.abs().amax((2, 3)) / 127.0)
    safe = torch.where(now > 0, now, torch.ones_like(now))[..., None, None]
    kept = torch.round(grid[pages, :, blk].float() * (old[..., None, None] / safe))
    put = torch.where(fresh, torch.round(v / safe).clamp(-127, 127), kept)
    scale[pages, :, blk] = now
    grid[pages, :, blk] = put.to(torch.int8)


def _values(codes, scale):
    return codes.float() * scale.repeat_interleave(BLOCK, 2)[..., None]


def _read_plain(codes, scale, at):
    pages, slot = at.unbind(1)
    return codes[pages, :, slot].float() * scale[pages, :, slot // BLOCK][..., None]


def _by_request(codes, scale, tables):
    """[requests, heads, positions, D] through the page tables."""
    r, n = tables.shape
    x = _values(codes[tables.view(-1).long()], scale[tables.view(-1).long()])
    p, h, page, d = x.shape
    return x.view(r, n, h, page, d).transpose(1, 2).reshape(r, h, n * page, d)


def _attend_plain(s):
    c = s["case"]
    hk, hq, d = c["k_heads"], c["q_heads"], c["head"]
    k = _by_request(s["codes"][0], s["scale"][0], s["tables"])
    v = _by_request(s["codes"][1], s["scale"][1], s["tables"])
    r, most = k.shape[0], max(c["new"], c["prompt"])
    i = torch.arange(most, device="cuda")
    rows = (s["first_row"][:, None] + i).clamp(max=s["q"].shape[0] - 1)
    q = s["q"][rows].float().view(r, most, hk, hq // hk, d).permute(0, 2, 3, 1, 4).reshape(r, hk, -1, d)
    score = (q @ k.transpose(2, 3)).view(r, hk, hq // hk, most, -1) / math.sqrt(d)
    here = (s["held"][:, None] + i)[:, :, None]
    at = torch.arange(score.shape[-1], device="cuda")
    seen = at <= here
    if c["window"]:
        seen &= at > here - c["window"]
    score = score.masked_fill(~seen[:, None, None], -math.inf)                         # (a token sees itself at least)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - top)
    total = p.sum(-1, keepdim=True)
    out = (p.view(r, hk, -1, p.shape[-1]) @ v).view(r, hk, hq // hk, most, d) / total
    lse = (top + torch.log(total))[..., 0]
    a, b = s["row_request"], s["row_index"]
    return out[a, :, :, b].reshape(-1, hq, d).to(s["q"].dtype), lse[a, :, :, b].reshape(-1, hq)


def _run_plain(s):
    op = s["case"]["op"]
    if op != "attend":
        _write_plain(s["codes"][0], s["scale"][0], s["k"], s["units"])
        _write_plain(s["codes"][1], s["scale"][1], s["v"], s["units"])
    if op != "store":
        return _attend_plain(s)
    t = s["k"].dtype
    return (_read_plain(s["codes"][0], s["scale"][0], s["seen_at"]).to(t),
            _read_plain(s["codes"][1], s["scale"][1], s["seen_at"]).to(t))


def run(state):
    s = state
    if not own:
        return _run_plain(s)
    op = s["case"]["op"]
    if op != "attend":
        s["cache"].write(s["k"], s["v"], s["plan"])
    if op != "store":
        return s["cache"].attend(s["q"], s["plan"], window=s["case"]["window"])
    return s["cache"].read(s["seen"], s["k"].dtype)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    c = case
    new, held = _lengths(c)
    hk, d = c["k_heads"], c["head"]
    token = 2 * hk * (d + 4 / BLOCK)                                                   # codes and scales of a token
    size = 4 if c.get("dtype") == "f32" else 2
    rows = sum(new)
    bytes_, flops = 0, 0
    if c["op"] != "attend":
        behind = sum(p % BLOCK for p, n in zip(held, new) if n)                        # tokens that their block holds
        bytes_ += rows * 2 * hk * d * size + (rows + behind) * token
        flops += 4 * rows * hk * d
    if c["op"] == "store":
        return {"bytes": bytes_ + (rows + behind) * 2 * hk * d * size, "flops": flops + 2 * (rows + behind) * hk * d}
    hq, w = c["q_heads"], c["window"]
    for n, p in zip(new, held):
        first = max(0, p + 1 - w) if w else 0
        bytes_ += (p + n - first) * token
        whole = max(0, min(n, w - p)) if w else n                                      # rows that see all before them
        flops += 4 * d * hq * (whole * p + whole * (whole + 1) // 2 + (n - whole) * w)
    return {"bytes": bytes_ + rows * hq * (4 * d + 4), "flops": flops}


# ------------------------------------------------------------------ the definitions in 64 bits
def _held64(parts):
    """What a head's block is given, part after part [(rows [n, D]), ...], as the values that it holds in the end.  The
    scale has 32 bits and a code is the nearest whole number of scales by a quotient of 32 bits: part of the definition."""
    scale, codes = torch.zeros((), device="cuda"), None
    for x in parts:
        x = x.float()
        bigger = torch.maximum(scale, x.abs().max() / 127.0)
        if float(bigger) == 0.0:
            fresh = torch.zeros_like(x)
        else:
            fresh = torch.round(x / bigger)
            if codes is not None:
                codes = torch.round(codes * (scale / bigger))
        codes, scale = fresh if codes is None else torch.cat([codes, fresh]), bigger
    return codes.double() * scale.double()


def _filled64(x):
    """The values held of x [n, heads, D] written in one call from position 0."""
    n, h, d = x.shape
    f = torch.zeros(-(-n // BLOCK) * BLOCK, h, d, device=x.device)
    f[:n] = x.float()
    f = f.view(-1, BLOCK, h, d)
    scale = (f.abs().amax((1, 3), keepdim=True) / 127.0)
    code = torch.where(scale > 0, f / scale, torch.zeros_like(f)).round()
    return (code.double() * scale.double()).view(-1, h, d)[:n]


def exact(case, seed):
    c = dict(case)
    new, held = _lengths(c)
    hk, d = c["k_heads"], c["head"]
    s = prepare(case, seed)
    # the same numbers again, as prepare() drew them
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    filled = [n + p for n, p in zip(new, held)] if c["op"] == "attend" else held
    old = [_rows(g, sum(filled), hk, d, torch.bfloat16) for _ in "kv"]
    rows = [s["k"], s["v"]]
    kept = [[], []]                                   # per request, [tokens, heads, D]
    a = b = 0
    for n, p, f in zip(new, held, filled):
        for which in (0, 1):
            x = old[which][a: a + f]
            if c["op"] == "attend":
                kept[which].append(_filled64(x))
                continue
            edge = p - p % BLOCK                      # whole blocks before; the last one goes on with the new rows
            fresh = rows[which][b: b + n]
            lead = min(n, BLOCK - p % BLOCK) if p % BLOCK else 0
            y = torch.zeros(p + n, hk, d, device="cuda", dtype=torch.float64)
            y[:edge] = _filled64(x[:edge])
            if lead:
                for h in range(hk):
                    y[edge: p + lead, h] = _held64([x[edge:, h], fresh[:lead, h]])
            y[p + lead:] = _filled64(fresh[lead:])
            kept[which].append(y)
        a += f
        b += n
    if c["op"] == "store":
        return tuple(torch.cat([y[p - p % BLOCK:] for y, p in zip(k, held)]) for k in kept)
    hq, w = c["q_heads"], c["window"]
    out = torch.empty(sum(new), hq, d, device="cuda", dtype=torch.float64)
    lse = torch.empty(sum(new), hq, device="cuda", dtype=torch.float64)
    b = 0
    for i, (n, p) in enumerate(zip(new, held)):
        for h in range(hq):
            k, v = kept[0][i][:, h * hk // hq], kept[1][i][:, h * hk // hq]
            for first in range(0, n, 2048):
                last = min(n, first + 2048)
                q = s["q"][b + first: b + last, h].double()
                z = torch.einsum("td,pd->tp", q, k[: p + last]) * d ** -0.5
                t, u = torch.arange(p + first, p + last, device="cuda"), torch.arange(p + last, device="cuda")
                away = t[:, None] - u[None]
                z[(away < 0) | (away >= w if w else away < 0)] = -math.inf
                lse[b + first: b + last, h] = torch.logsumexp(z, 1)
                out[b + first: b + last, h] = torch.einsum("tp,pd->td", torch.softmax(z, 1), v[: p + last])
        b += n
    return out, lse

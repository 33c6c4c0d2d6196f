"""From a calibrated layer to adapters trained over its codes, and attention over an 8-bit cache: one attention block.

    python examples/adapt_attention_input.py [--hidden 1024] [--steps 30]

The q, k and v projections of a block are quantized (W3, groups of 128) by the solver from calibration activations, and
laid out for multiplication.  Two groups of requests then train an adapter each, so that the block's normed and rotated
queries and keys, and its values, come back to those of the unquantized weights: forward through the codes and the
adapters, inputs kept in 8 bits, backward through the rotation, the norm and the codes.  At the end one new token of every
request runs through the trained adapters, beside one that has none: the prompts' keys and values, kept in 8 bits, are
attended over by the prompts themselves and by the new tokens.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2605_11222_b200 import adapt, binding as B, kvcache, workloads as wl  # noqa: E402

HEAD, GROUP, BITS, EPS, PAGE = 64, 128, 3, 1e-6, 32


def quantize(spec, W, X):
    """Solver and local search on one weight matrix -> the packed layer."""
    sol = B.Solver(spec.d_in, W.shape[0], T_max=spec.T)
    sol.hessian_reset()
    sol.hessian_accumulate(X)
    sol.factor(rho=spec.rho())
    codes, scale, zero, _ = sol.quantize_layer(W, BITS, GROUP)
    sol.local_search(W, BITS, GROUP, codes, scale, zero)
    assert sol.last_device_status() == B.OK
    return adapt.QuantLinear(codes, scale, zero, BITS, GROUP)


class AttentionInput:
    """q, k, v projections on codes with adapters, and the norm and rotation of queries and keys."""

    def __init__(self, layers, banks, heads, kv_heads, positions=4096, dev="cuda"):
        self.layers, self.banks, self.heads, self.kv_heads = layers, banks, heads, kv_heads
        self.wq = torch.ones(HEAD, dtype=torch.bfloat16, device=dev)
        self.wk = torch.ones(HEAD, dtype=torch.bfloat16, device=dev)
        ang = torch.arange(positions, device=dev)[:, None] * 1e4 ** (-torch.arange(0, HEAD, 2, device=dev) / HEAD)
        self.cos, self.sin = ang.cos(), ang.sin()

    def forward(self, x, plan, pos):
        (q, hq), (k, hk), (v, hv) = [l.forward(x, b, plan) for l, b in zip(self.layers, self.banks)]
        t = x.shape[0]
        q, k = q.view(t, self.heads, HEAD), k.view(t, self.kv_heads, HEAD)
        qr, kr = adapt.qk_norm_rope(q, k, self.wq, self.wk, self.cos, self.sin, pos, EPS)
        return (qr, kr, v), (q, k, (hq, hk, hv), adapt.Checkpoint.save(x), plan, pos)

    def backward(self, dqr, dkr, dv, saved):
        """Gradients of x and of every bank's (down, up)."""
        q, k, h, kept, plan, pos = saved
        t = q.shape[0]
        dq, dk, _, _ = adapt.qk_norm_rope_backward(q, k, self.wq, self.wk, self.cos, self.sin, pos, dqr, dkr, EPS)
        dx, grads = 0, []
        for layer, bank, hh, dy in zip(self.layers, self.banks, h, (dq.view(t, -1), dk.view(t, -1), dv)):
            d, u = layer.grad_input(dy, bank, plan)
            dx = dx + d
            grads.append(adapt.adapter_grads(bank, plan, kept, hh, dy, u))
        return dx, grads


def prompts_and_a_token(block, x, x_new, lengths, plan, new, pos, dev):
    """Attention of the prompts' rows, then of one token behind each, over keys and values in 8 bits."""
    need = [-(-(n + 1) // PAGE) for n in lengths]
    tables, at = [], 0
    for n in need:
        tables.append(list(range(at, at + n)) + [0] * (max(need) - n))
        at += n
    cache = kvcache.KVCache(at, block.kv_heads, HEAD, PAGE, dev)
    step = kvcache.CachePlan([1] * len(lengths), lengths, tables, block.heads // block.kv_heads, dev)
    prompt = kvcache.CachePlan(lengths, [0] * len(lengths), step.tables, step.group)
    out = []
    for rows, where, requests, positions in ((x, prompt, plan, pos), (x_new, step, new, step.held.clone())):
        (q, k, v), _ = block.forward(rows, requests, positions)
        cache.write(k, v.view_as(k), where)
        out.append(cache.attend(q, where)[0])
    adapt.check_device_status(dev)
    return out


def main(hidden=1024, steps=30, rank=16, rows=384, dev="cuda:0", quiet=False):
    torch.manual_seed(0)
    heads, kv_heads, adapters = hidden // HEAD, max(1, hidden // HEAD // 4), 2
    spec = wl.small_case(hidden, heads * HEAD, 4096, T=40, seed=11)
    X = wl.gen_x_chunk(spec, 0, dev)
    weights = [(torch.randn(n * HEAD, hidden, device=dev) * 0.02).contiguous() for n in (heads, kv_heads, kv_heads)]
    layers = [quantize(spec, W, X) for W in weights]
    banks = []
    for W in weights:
        down = (torch.rand(adapters, rank, hidden, device=dev) * 2 - 1) / math.sqrt(hidden)
        banks.append(adapt.AdapterBank(down.bfloat16(), torch.zeros(adapters, rank, W.shape[0], dtype=torch.bfloat16, device=dev),
                                       torch.full((adapters,), 2.0, device=dev)))
    block = AttentionInput(layers, banks, heads, kv_heads, dev=dev)

    # two groups of requests, each with its adapter, one request without; the inputs of the last calibration rows
    lengths = [rows // 2, rows // 4, rows - rows // 2 - rows // 4]
    plan = adapt.RequestPlan(lengths, [0, 1, -1], adapters, dev)
    pos = torch.cat([torch.arange(n) for n in lengths]).int().to(dev)
    x = X[:rows].contiguous()
    q, k, v = [(x.float() @ W.T).bfloat16() for W in weights]
    want = (*adapt.qk_norm_rope(q.view(rows, heads, HEAD), k.view(rows, kv_heads, HEAD), block.wq, block.wk, block.cos,
                                block.sin, pos, EPS), v)
    master = [[p.float() for p in (b.down, b.up)] for b in banks]
    moments = [[(torch.zeros_like(p), torch.zeros_like(p)) for p in m] for m in master]
    losses = []
    on = (plan.row_adapter >= 0)[:, None]
    for step in range(1, steps + 1):
        got, saved = block.forward(x, plan, pos)
        diff = [(g.float() - w.float()).view(rows, -1) * on for g, w in zip(got, want)]
        losses.append(sum(float(d.square().mean()) for d in diff))
        dqr, dkr, dv = [(2.0 * d / d.numel() * rows).bfloat16() for d in diff]
        dx, grads = block.backward(dqr.view_as(got[0]), dkr.view_as(got[1]), dv, saved)
        for bank, m, mo, g in zip(banks, master, moments, grads):            # Adam on fp32 copies
            for p, live, (a, b), gr in zip(m, (bank.down, bank.up), mo, g):
                a.mul_(0.9).add_(gr.float(), alpha=0.1)
                b.mul_(0.99).addcmul_(gr.float(), gr.float(), value=0.01)
                p -= 2e-3 * (a / (1 - 0.9 ** step)) / ((b / (1 - 0.99 ** step)).sqrt() + 1e-8)
                live.copy_(p)
    adapt.check_device_status(dev)
    if not quiet:
        print(f"error of the block's outputs, adapted rows: {losses[0]:.5f} -> {losses[-1]:.5f} in {steps} steps")

    # decoding: a new token of every request
    new = adapt.RequestPlan([1, 1, 1], [0, 1, -1], adapters, dev)
    (qr, kr, v1), _ = block.forward(X[rows: rows + 3].contiguous(), new, torch.tensor(lengths, dtype=torch.int32, device=dev))
    alone = layers[0].forward(X[rows + 2: rows + 3].contiguous())[0]
    again = layers[0].forward(X[rows: rows + 3].contiguous(), banks[0], new)[0]
    same = torch.equal(again[2], alone[0])
    prompt_out, token_out = prompts_and_a_token(block, x, X[rows: rows + 3].contiguous(), lengths, plan, new, pos, dev)
    if not quiet:
        print(f"attention of the prompts {tuple(prompt_out.shape)} and of the tokens {tuple(token_out.shape)} over the 8-bit cache")
        print(f"decoded 3 tokens, q {tuple(qr.shape)}, k {tuple(kr.shape)}; the one without an adapter is the layer's alone: {same}")
    return losses, dx, same


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--hidden", type=int, default=1024)
    ap.add_argument("--steps", type=int, default=30)
    a = ap.parse_args()
    main(a.hidden, a.steps)

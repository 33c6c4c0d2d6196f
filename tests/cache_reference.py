"""The cache of keys and values and attention over it, from their definitions, for the tests: scales and codes in 32 bits on
the host as the definition has them, attention in 64 bits."""
import math

import numpy as np
import torch

BLOCK = 16


class ReferenceCache:
    """Blocks as dictionaries: (page, block of the page) -> per head scale [heads] fp32 and codes [heads, 16, D]."""

    def __init__(self, heads, dim, page):
        self.heads, self.dim, self.page, self.blocks = heads, dim, page, {}

    def _put(self, which, key, first, rows):
        """rows [n, heads, D] fp32 at slots first .. of a block."""
        n = rows.shape[0]
        scale, codes = self.blocks.get((which, *key), (np.zeros(self.heads, np.float32), np.zeros((self.heads, BLOCK, self.dim), np.float32)))
        if first == 0:
            scale, codes = np.zeros(self.heads, np.float32), np.zeros_like(codes)
        x = rows.transpose(1, 0, 2).astype(np.float32)
        codes = codes.copy()
        now = scale.copy()
        for h in range(self.heads):
            top = np.abs(x[h]).max() if np.isfinite(x[h]).all() else np.float32(np.inf)
            if not top < 2.0 ** 40 or not scale[h] == scale[h]:
                now[h], codes[h] = np.nan, 0
                continue
            add = np.float32(0) if top < 2.0 ** -40 else np.float32(top) * (np.float32(1) / np.float32(127))
            now[h] = max(scale[h], add)
            if now[h] == 0:
                codes[h, first: first + n] = 0
                continue
            if now[h] != scale[h]:
                codes[h, :first] = np.rint(codes[h, :first] * np.float32(scale[h] / now[h]))
            codes[h, first: first + n] = np.rint(x[h] / now[h])
        self.blocks[(which, *key)] = (now, codes)

    def write(self, k, v, lengths, held, tables):
        row = 0
        for i, n in enumerate(lengths):
            p, end = held[i], held[i] + n
            while held[i] >= 0 and p < end:
                stop = min(end, p - p % BLOCK + BLOCK)
                at = row + p - held[i]
                for which, x in (("k", k), ("v", v)):
                    self._put(which, (tables[i][p // self.page], p % self.page // BLOCK), p % BLOCK,
                              x[at: at + stop - p].float().cpu().numpy())
                p = stop
            row += n

    def token(self, which, pages, p):
        scale, codes = self.blocks[(which, pages[p // self.page], p % self.page // BLOCK)]
        return scale[:, None].astype(np.float64) * codes[:, p % BLOCK].astype(np.float64)

    def sequence(self, which, pages, n):
        """[n, heads, D] in 64 bits."""
        if n <= 0:
            return torch.zeros(0, self.heads, self.dim, dtype=torch.float64)
        return torch.from_numpy(np.stack([self.token(which, pages, p) for p in range(n)]))

    def rows(self, which, lengths, held, tables):
        out = []
        for i, n in enumerate(lengths):
            if held[i] < 0:
                out.append(torch.zeros(n, self.heads, self.dim, dtype=torch.float64))
            else:
                out += [torch.from_numpy(self.token(which, tables[i], p))[None] for p in range(held[i], held[i] + n)]
        return torch.cat(out) if out else torch.zeros(0, self.heads, self.dim, dtype=torch.float64)


def attend64(q, sequences, lengths, held, group, scale, window=0):
    """q [rows, heads * group, D]; sequences[i] = (k, v) [tokens, heads, D].  Returns out, lse and the tolerances of both for
    a kernel whose weights are rounded to fp16, whose sums have 32 bits and whose result is bf16:
     - the result: 2^-8 |out|;
     - every weight: 2^-11 of itself, independent, so six standard deviations are 6 / sqrt(3) 2^-11 sqrt(sum (w v)^2),
       and below the fp16 numbers of full precision 2^-25 of the largest weight's unit, at random again;
     - a score: at most 16 steps of the product that lose 2^-23 of the sum of magnitudes each, and five further roundings
       of it and of its power of two (2^-22 each, of numbers as large as the score's and the scales' logarithms).  An error d
       of the scores moves the result by at most 2 d sum w |v|;
     - the sum over positions: 2^-18 sum w |v| (see the projections' tests)."""
    rows, hq, d = q.shape
    out = torch.zeros(rows, hq, d, dtype=torch.float64)
    lse = torch.full((rows, hq), -math.inf, dtype=torch.float64)
    t_out, t_lse = torch.zeros_like(out), torch.zeros_like(lse)
    q = q.double().cpu()
    row = 0
    for i, n in enumerate(lengths):
        if held[i] >= 0 and n > 0:
            k, v = sequences[i]
            for h in range(hq):
                kk, vv = k[:, h // group], v[:, h // group]
                qq = q[row: row + n, h]
                z = (qq @ kk.T) * scale
                size = (qq.abs() @ kk.abs().T) * scale
                at = torch.arange(n)[:, None] + held[i] - torch.arange(kk.shape[0])[None]
                away = (at < 0) | ((at >= window) if window else torch.zeros_like(at, dtype=torch.bool))
                z = z.masked_fill(away, -math.inf)
                w = torch.softmax(z, 1)
                o = w @ vv
                out[row: row + n, h] = o
                lse[row: row + n, h] = torch.logsumexp(z, 1)
                seen = torch.where(away, torch.zeros_like(size), size).amax(1)
                biggest = torch.where(away, torch.zeros_like(z), z.abs()).amax(1)
                dz = 16 * 2.0 ** -23 * seen + 5 * 2.0 ** -22 * (1.45 * biggest + 64)
                mean = w @ vv.abs()
                square = ((w ** 2) @ (vv ** 2)).sqrt()
                tiny = 2.0 ** -25 * 6 * vv.abs().amax(0) * w.amax(1, keepdim=True) * math.sqrt(kk.shape[0])
                t_out[row: row + n, h] = 2.0 ** -8 * o.abs() + 6 / math.sqrt(3) * 2.0 ** -11 * square + tiny + \
                    (2 * dz[:, None] + 2.0 ** -18) * mean
                t_lse[row: row + n, h] = dz + 2.0 ** -18 + 2.0 ** -22 * lse[row: row + n, h].abs()
        row += n
    return out, lse, t_out, t_lse

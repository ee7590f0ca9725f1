"""Prompt attention in 64 bits, with the tolerance of a kernel whose weights and outputs are rounded once each.

With weights p (1 + e), |e| <= u, the output is off by sum p e (v - o) / sum p: at most u (A + |o|), A = sum p |v| / sum p.  u counts:
  the rounding of the weights, half a step of their type (2^-8 bf16, 2^-11 fp16; fp16 weights below 2^-14 round to a grid of 2^-24, where
  the largest is at least 1: 2^-25 n max |v| in all);
  the logits, summed in 32 bits: 128 additions and three products, 2^-24 each of sum |q k|, and 2^-22 for the exponential;
  the sums over n keys, at most n / 8 additions in a row (a step of the matrix instruction takes 16 keys), joins and rescalings beside them;
and the output's own half step."""
import math

import torch

HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def attention(q, k, v, before, lens, cached, sm_scale, out_type, prefix_type=torch.float16):
    """(value, tolerance) [tokens, heads, 128] in 64 bits; rows behind the last sequence are zero."""
    hq, r = q.shape[1], q.shape[1] // k.shape[1]
    out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    tol = torch.zeros_like(out)
    a = p = 0
    for n, c in zip(lens, cached):
        for h in range(hq if n else 0):
            K, V = (torch.cat(([x[p:p + c, h // r].double()] if c else []) + [y[a:a + n, h // r].double()]) for x, y in zip(before, (k, v)))
            Q = q[a:a + n, h].double()
            hidden = torch.ones((n, n), dtype=torch.bool, device=q.device).triu(1)
            logits = (Q @ K.t().contiguous()) * sm_scale
            logits[:, c:].masked_fill_(hidden, -math.inf)
            weight = torch.softmax(logits, -1)
            o, size = weight @ V, weight @ V.abs()
            off = 132 * 2.0 ** -24 * sm_scale * (Q.abs() @ K.abs().t().contiguous())
            off[:, c:].masked_fill_(hidden, 0.0)
            u = max(HALF[k.dtype], HALF[prefix_type] if c else 0.0) + off.amax(-1, keepdim=True) + 2.0 ** -22 + (c + n) / 8 * 2.0 ** -23 + 16 * 2.0 ** -24
            out[a:a + n, h] = o
            tol[a:a + n, h] = HALF[out_type] * o.abs() + 2.0 ** -25 + u * (size + o.abs())
            if torch.float16 in (k.dtype, prefix_type if c else k.dtype):
                tol[a:a + n, h] += 2.0 ** -25 * (c + n) * V.abs().amax()
        a, p = a + n, p + c
    return out, tol


KEYS = {32: 32, 128: 64, 256: 64}     # keys of a tile, by rows


def plan_of(rows, most, lens, cached, group):
    """A plan with tiles of `rows` rows and ranges of at most `most` tiles of keys."""
    import numpy as np

    from paper_2605_17170_amd import tkv
    items, cuts, slot, a, p = [], [], 0, 0, 0
    for n, c in zip(lens, cached):
        for row in range(0, n * group, rows):
            see = (min(row + rows, n * group) - 1) // group + 1
            keys = -(-c // KEYS[rows]) + -(-see // KEYS[rows])
            parts = -(-keys // most)
            if parts > 1:
                cuts.append([a, n, row, slot, parts])
            for k in range(parts):
                items.append([a, n, p, c, row, keys * k // parts, keys * (k + 1) // parts, slot if parts > 1 else -1, k, parts] + 6 * [0])
                slot += parts > 1
        a, p = a + n, p + c
    for k, cut in enumerate(cuts):
        items[k][10:15] = cut
    return tkv.PrefillPlan(np.array(items, np.int32).reshape(-1, 16), slot, rows, len(cuts))

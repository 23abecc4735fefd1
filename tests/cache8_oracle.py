"""The 8-bit cache, attention over it, and the choice of a token from their definitions, in 64 bits (test infrastructure).

torch is used for arrays and elementary arithmetic only; nothing here comes from the package.
"""
import math

import torch

BLOCK = 64


def held(x, heads):
    """(values, codes or None, scales) that a cache holds of bf16 rows [n, heads * d]: values fp32 [n, heads, d]; scales fp32 [blocks, heads]"""
    n, d = x.shape[0], x.shape[1] // heads
    x = x.view(n, heads, d)
    full = n // BLOCK
    out = x.float().clone()
    scales = torch.empty(full, heads)
    codes = torch.zeros(full * BLOCK, heads, d)
    for b in range(full):
        for h in range(heads):
            t = x[b * BLOCK:(b + 1) * BLOCK, h].double()
            if not torch.isfinite(t).all():
                scales[b, h] = math.nan
                out[b * BLOCK:(b + 1) * BLOCK, h] = math.nan
                continue
            s = (torch.clamp(t.abs().max(), min=2.0 ** -100) / 127).float()
            # to the nearest, ties to even; the quotient of two short numbers is no near-tie in 64 bits (+ 0: a whole number has no -0)
            q = torch.round(t / s.double()) + 0.0
            scales[b, h], codes[b * BLOCK:(b + 1) * BLOCK, h] = s, q.float()
            out[b * BLOCK:(b + 1) * BLOCK, h] = (q * s.double()).float()
    return out, codes, scales


def attention(q, k, v, heads):
    """fp64 [rows, heads, d] of bf16 q [rows, heads * d] over values k, v [n, kv_heads, d]; and what bounds its error: sum of p |v|, and the largest
    sum of |q| |k| / sqrt(d) of a row and head"""
    rows, n, kv = q.shape[0], k.shape[0], k.shape[1]
    d = q.shape[1] // heads
    q, k, v = q.double().view(rows, heads, d), k.double(), v.double()
    o, size, reach = (torch.zeros(rows, heads, d, dtype=torch.float64, device=q.device) for _ in range(3))
    for h in range(heads):
        kh, vh = k[:, h // (heads // kv)], v[:, h // (heads // kv)]
        for i in range(rows):
            see = n - rows + i + 1
            s = kh[:see] @ q[i, h] / math.sqrt(d)
            p = torch.exp(s - s.max())
            p = p / p.sum()
            o[i, h] = p @ vh[:see]
            size[i, h] = p @ vh[:see].abs()
            reach[i, h] = (kh[:see].abs() @ q[i, h].abs()).max() / math.sqrt(d)
    return o, size, reach


def attention_bound(o, size, reach, d, n, p_rounding):
    """How far a kernel may be from `o`: its own rounding (bf16: half a step, 2^-8 of the value), a probability rounded by p_rounding of itself,
    and fp32 arithmetic: a score of d products in any order is off by (d + 2) 2^-24 of the sum of their magnitudes (and the products with the scales by
    three roundings more), which an exponential turns into as much of its value, in the numerator and in the denominator; sums over n keys by n 2^-24."""
    c = p_rounding + 2 * (d + 6) * 2.0 ** -24 * reach + 2 * n * 2.0 ** -24 + 2.0 ** -20
    return 2.0 ** -8 * o.abs() + (1 + 2.0 ** -8) * c * size


def choose(logits, counts, repetition, presence, frequency, bias, allowed):
    """values in fp64 (each input as it is), -inf where not allowed, and whether a token may be chosen"""
    x = logits.double()
    R, V = x.shape
    c = torch.zeros(R, V) if counts is None else counts.double().expand(R, V)
    y = torch.where(x > 0, x / repetition, x * repetition) - (frequency * c + presence)
    y = torch.where(c > 0, y, x)
    if bias is not None:
        y = y + bias.double()
    may = torch.ones(R, V, dtype=torch.bool)
    if allowed is not None:
        word = allowed.expand(R, allowed.shape[-1]).long()[:, torch.arange(V) // 32]
        may = (word >> (torch.arange(V) % 32) & 1).bool()
    return torch.where(may, y, -math.inf), may

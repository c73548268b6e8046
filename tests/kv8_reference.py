"""Rows held in 8 bits, restated in 64 bits: e4m3 codes with the least power-of-two
scale for every SCALE_ROWS slots of a page and head with which the largest finite
element is at most 448."""
import math

import torch

SCALE_ROWS = 8
LEAST = -100


def scale_of(size):
    """Scales (float64) for the largest sizes `size` (float64)."""
    e = torch.full_like(size, LEAST)
    on = size > 0
    x = torch.ceil(torch.log2(size[on] / 448.0))
    # (the logarithm may be a digit off at a border)
    x = torch.where(torch.exp2(x - 1) * 448.0 >= size[on], x - 1, x)
    x = torch.where(torch.exp2(x) * 448.0 < size[on], x + 1, x)
    e[on] = x.clamp(min=LEAST)
    return torch.exp2(e)


def nearest(x):
    """e4m3 values nearest to x (float64, |x| <= 448 or NaN), ties to even."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def blocks_of(fills, page):
    """Slices of a sequence's rows that share blocks, for its pages' fills."""
    out, at = [], 0
    for f in fills:
        out += [(at + b, at + min(b + SCALE_ROWS, f)) for b in range(0, f, SCALE_ROWS)]
        at += f
    return out


def held(rows, blocks):
    """What rows [n, heads, d] (float64) in these blocks are held as, and each row's
    scale [n, heads]."""
    out, scales = torch.empty_like(rows), rows.new_empty(rows.shape[:2])
    for a, b in blocks:
        x = rows[a:b]
        x = torch.where(x.isinf(), torch.full_like(x, math.nan), x)
        # (what rounds to 2^128 would be an infinity)
        x = x.clamp(-240 * 2.0 ** 120, 240 * 2.0 ** 120)
        s = scale_of(torch.nan_to_num(x.abs(), nan=0.0).amax((0, 2)))
        out[a:b] = nearest(x / s[None, :, None]) * s[None, :, None]
        scales[a:b] = s
    return out, scales


def attention(q, k, v, scale, keep=None):
    """(outputs, sum of |weight * value|, largest |logit| sum of products) of q [m, hq, d]
    over rows k, v [n, hkv, d]; keep [m, n]."""
    m, hq, d = q.shape
    g = hq // k.shape[1]
    kk, vv = k.double().repeat_interleave(g, 1), v.double().repeat_interleave(g, 1)
    s = torch.einsum("mhd,nhd->hmn", q.double(), kk) * scale
    size = torch.einsum("mhd,nhd->hmn", q.double().abs(), kk.abs()) * scale
    if keep is not None:
        s = s.masked_fill(~keep[None], -math.inf)
        size = size.masked_fill(~keep[None], 0.0)
    w = torch.softmax(s, -1)
    return (torch.einsum("hmn,nhd->mhd", w, vv), torch.einsum("hmn,nhd->mhd", w, vv.abs()),
            size.amax(-1).transpose(0, 1))


def token_budget(ref, weighted, logits, d):
    """Most that a single token's fp32 output may be off: each weight's rounding to fp16
    (half a step of 11 bits, 2^-11; the normaliser sums the rounded ones: twice), the
    exponential's argument (fp32 sums of d products and two factors, 2^-24 each, of
    sizes up to `logits`, twice; the maximum's subtraction, of arguments up to
    1.45 logits), the exponential itself (2^-21) and fp32 sums (2^-16)."""
    return weighted * (2.0 ** -10 + (2.0 * (d + 8) * 2.0 ** -24 * logits)[..., None] + 2.0 ** -16) + 1e-37

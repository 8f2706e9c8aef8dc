"""How far a result of the attention operators may be from the exact one where rows see
many keys: element by element, and over all elements together."""
from __future__ import annotations

import torch
from attn_util import TINY, UNIT, attend

# a row's largest weight stands at no less than this before it is rounded to the type
LEAST_TOP = {torch.bfloat16: 1.0, torch.float16: 2.0 ** 8}


def bound(q, k, v, scale, seen):
    """q [n, H, D], k and v [m, G, D], seen [n, m] bool, every row with a key.  Returns the exact
    out [n, H, D], the largest error of each element, and of the root mean square of all.

    Element by element, as in attn_util: a weight's relative error is that of its score
    (D + 4 roundings of 2^-24 against the sum of the products' sizes, 2^-22 of the score) and a few
    2^-22 of the exponential; it is rounded to the type (relative UNIT); a weight below the type's
    normal range is off by TINY instead, against a row sum of at least LEAST_TOP; sums of m
    terms add m 2^-24; and the result is rounded once.

    Together: roundings of different weights are independent, so that their part in an element is
    UNIT / sqrt(3) of the root of the sum of (p v)^2.  For values without a mean, of equal size,
    that root and the result itself have the same root mean square.  With the result's own
    rounding, of the same size, that is 0.82 UNIT of it; the limit is 2 UNIT, and m 2^-24 for the sums."""
    dtype = q.dtype
    n, H, D = q.shape
    m, G = k.shape[:2]
    u = UNIT[dtype]
    out = attend(q, k, v, scale, seen)[0]
    qd, kd, vd = q.double().view(n, G, H // G, D), k.double(), v.double()
    s = torch.einsum("nghd,mgd->nghm", qd, kd) * scale
    size = torch.einsum("nghd,mgd->nghm", qd.abs(), kd.abs()) * abs(scale)
    mask = seen[:, None, None, :]
    off = torch.where(mask, size * (D + 4) * 2.0 ** -24 + s.abs() * 2.0 ** -22, 0.0).amax(-1)
    p = torch.softmax(s.masked_fill(~mask, float("-inf")), -1)
    mean = torch.einsum("nghm,mgd->nghd", p, vd.abs())
    top = vd.abs().amax((0, 2))[None, :, None, None]
    rel = 1.05 * u + 2.0 * (off[..., None] * 1.05 + 8 * 2.0 ** -22 + m * 2.0 ** -24)
    lim = mean * rel + TINY[dtype] * (1 + m * top / LEAST_TOP[dtype])
    lim = lim.reshape(n, H, D) + out.abs() * u * 1.05 + 1e-30
    return out, lim, float(out.square().mean().sqrt()) * (2 * u + m * 2.0 ** -24)


def misses(got, want, lim, rms):
    """What is wrong with a result, or None."""
    err = (got.double() - want).abs()
    if not bool((err <= lim).all()):
        return f"{int((~(err <= lim)).sum())} of {err.numel()} elements off, by up to {float((err / lim).max())} of their limit"
    if not float(err.square().mean().sqrt()) <= rms:
        return f"root mean square off by {float(err.square().mean().sqrt())}, limit {rms}"
    return None

"""Attention from its definition in 64 bits, with a bound on how far a result of
the operators may be from it: what the tests of the attention operators use."""
from __future__ import annotations

import math

import torch

UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}      # half a spacing, relative: 8 and 11 significant bits
TINY = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}    # half the smallest spacing


def attend(q, k, v, scale, seen):
    """q [n, H, D], k and v [m, G, D], seen [n, m] bool.  Returns the exact out
    [n, H, D] and lse [n, H], and the largest error of each that rounding allows.

    A score is a sum of D products in 32 bits, scaled into powers of two: off by
    at most (D + 4) 2^-24 of the sum of the products' sizes and 2^-22 of itself.  Its
    exponential carries that as a relative error, plus a few 2^-22 of the
    exponential itself; the weights are then rounded to the type (relative UNIT,
    absolute TINY each, against a row sum of at least 2^-8: a row's largest
    weight may stand at 2^-8 .. 2^8), the accumulation adds m 2^-24 at most,
    and the result is rounded once."""
    dtype = q.dtype
    n, H, D = q.shape
    m, G = k.shape[:2]
    qd = q.double().view(n, G, H // G, D)
    clean = seen.any(0)                                     # what no row sees has no influence
    kd, vd = (torch.where(clean[:, None, None], x.double(), 0.0) for x in (k, v))
    s = torch.einsum("nghd,mgd->nghm", qd, kd) * scale
    size = torch.einsum("nghd,mgd->nghm", qd.abs(), kd.abs()) * abs(scale)
    s = torch.where(seen[:, None, None, :], s, -math.inf)
    some = seen.any(1)[:, None, None]
    lse = torch.logsumexp(s, -1) if m else torch.full((n, G, H // G), -math.inf, dtype=torch.float64, device=q.device)
    p = torch.exp(s - torch.where(some, lse, 0.0)[..., None])
    out = torch.where(some[..., None], torch.einsum("nghm,mgd->nghd", p, vd), 0.0)
    u = UNIT[dtype]
    if m:
        seen_size = torch.where(seen[:, None, None, :], size, 0.0)
        off = (seen_size * (D + 4) * 2.0 ** -24 + torch.where(seen[:, None, None, :], s, 0.0).abs() * 2.0 ** -22).amax(-1)
        top = torch.where(seen[:, :, None, None].expand(-1, -1, G, D), vd.abs(), 0.0).amax(1)[:, :, None, :]
    else:
        off = torch.zeros((n, G, H // G), dtype=torch.float64, device=q.device)
        top = torch.zeros((n, G, 1, D), dtype=torch.float64, device=q.device)
    mean = torch.einsum("nghm,mgd->nghd", p.nan_to_num(0.0), vd.abs())
    rel = 1.05 * u + 2.0 * (off[..., None] * 1.05 + 8 * 2.0 ** -22 + m * 2.0 ** -24)
    lim = mean * rel + out.abs() * u * 1.05 + TINY[dtype] * (1 + m * 2.0 ** 8 * top) + 1e-30
    lse_lim = off * 1.05 + 2.0 ** -20 + m * 2.0 ** -24 + torch.where(some, lse, 0.0).abs() * 2.0 ** -22
    return out.reshape(n, H, D), lse.reshape(n, H), lim.reshape(n, H, D), lse_lim.reshape(n, H)


def assert_within(got, want, lim, what=""):
    got = got.double()
    bad = ~((got - want).abs() <= lim) & ~((got == want) & ~torch.isfinite(want))
    if bad.any():
        at = bad.nonzero()[0].tolist()
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} off, first at {at}: got "
                             f"{got[tuple(at)].item()}, want {want[tuple(at)].item()} within {lim[tuple(at)].item()}")


def causal_mask(n, m, device):
    """Query i of the last n of m tokens sees the keys up to its own."""
    return torch.arange(m, device=device)[None] <= torch.arange(n, device=device)[:, None] + (m - n)


def randn(gen, shape, dtype, spread=1.0):
    return (torch.randn(shape, generator=gen, device=gen.device) * spread).to(dtype)

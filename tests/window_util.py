"""What the tests of windows and of caches in 8 bits share: masks, the definition of
the codes by a table of all of them, and a model of the cache that keeps whole pools."""
from __future__ import annotations

import math

import numpy as np
import torch

BLOCK = 16


def near_mask(n, m, window, sinks, device):
    """Query i of the last n of m tokens sees the last `window` keys up to its own, and the first `sinks`."""
    p = torch.arange(n, device=device)[:, None] + (m - n)
    j = torch.arange(m, device=device)[None]
    return (j <= p) & ((j > p - window) | (j < sinks))


def _values():
    """The value of every code: 1 bit of sign, 4 of exponent (from 2^-6 on), 3 of mantissa; 0x7f is NaN."""
    v = []
    for c in range(128):
        e, m = c >> 3, c & 7
        v.append(math.nan if c == 127 else m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
    return np.array(v + [-x for x in v])


VALUES = _values()


def codes_of(x):
    """Codes of numbers, by search: the nearest, of two the even one; at most 448; NaN where not finite."""
    x = np.asarray(x, np.float64)
    with np.errstate(invalid="ignore"):
        top = VALUES[:127]
        a = np.abs(x)
        hi = np.searchsorted(top, a).clip(0, 126)
        lo = (hi - 1).clip(0)
        near = np.where((a - top[lo] < top[hi] - a) | ((a - top[lo] == top[hi] - a) & (lo % 2 == 0)), lo, hi)
    near = np.where(np.isfinite(x), near, 127)
    return (near | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def scale_for(top):
    """The least power of two from 2^-126 to 2^119 that takes `top` to 448 at most."""
    e = -126
    while e < 119 and top > 448 * 2.0 ** e:
        e += 1
    return 2.0 ** e


def same_codes(got, want):
    """Equal codes; those of NaN whatever their sign."""
    nan = (got & 127 == 127) & (want & 127 == 127)
    return bool(((got == want) | nan).all())


class Model8:
    """The cache in 8 bits from its definition, one sequence, page and block after another;
    pools as the cache has them, with what nobody wrote."""

    def __init__(self, cache):
        self.page, self.per = cache.k_pages.shape[2], cache.table.shape[1]
        self.pools = [x.view(torch.uint8).cpu().numpy().copy() for x in (cache.k_pages, cache.v_pages)]
        self.scales = [x.double().cpu().numpy().copy() for x in (cache.k_scales, cache.v_scales)]
        self.seqs = [[] for _ in range(cache.table.shape[0])]
        self.length = [0] * len(self.seqs)
        self.refs = [0] * len(self.pools[0])

    def take(self):
        p = self.refs.index(0)
        self.refs[p] = 1
        return p

    def append(self, seqs, counts, k, v):
        """k, v: float64 [tokens, heads, dim]."""
        at, work = 0, []
        for s, n in zip(seqs, counts):
            part = self.length[s] % self.page
            if n and part and self.refs[self.seqs[s][-1]] > 1:
                old, new = self.seqs[s][-1], self.take()
                for pool, scales in zip(self.pools, self.scales):
                    pool[new][:, :part] = pool[old][:, :part]
                    scales[new][:, :-(-part // BLOCK)] = scales[old][:, :-(-part // BLOCK)]
                self.refs[old] -= 1
                self.seqs[s][-1] = new
            while len(self.seqs[s]) * self.page < self.length[s] + n:
                self.seqs[s].append(self.take())
            work.append((s, n, at))
            at += n
        # (every page is copied before any is written)
        for s, n, at in work:
            self.write(s, n, [x[at:at + n] for x in (k, v)])
            self.length[s] += n

    def write(self, s, n, rows):
        old = self.length[s]
        for b in range(old // BLOCK, -(-(old + n) // BLOCK) if n else 0):
            lo, hi = max(old, b * BLOCK), min(old + n, b * BLOCK + BLOCK)
            page, at = self.seqs[s][b * BLOCK // self.page], b * BLOCK % self.page
            for pool, scales, x in zip(self.pools, self.scales, rows):
                for g in range(pool.shape[1]):
                    new = x[lo - old:hi - old, g]
                    fine = np.abs(new[np.isfinite(new)])
                    need = scale_for(fine.max() if fine.size else 0.0)
                    before = lo - b * BLOCK
                    was = scales[page, g, at // BLOCK]
                    scale = max(was, need) if before else need
                    if before and scale > was:
                        share = float(np.float32(was) / np.float32(scale))
                        kept = np.float32(VALUES[pool[page, g, at:at + before]]) * np.float32(share)
                        pool[page, g, at:at + before] = codes_of(kept)
                    with np.errstate(invalid="ignore"):
                        pool[page, g, at + before:at + hi - b * BLOCK] = codes_of(np.float32(new) / np.float32(scale))
                    scales[page, g, at // BLOCK] = scale

    def fork(self, src, dst):
        for a, b in zip(src, dst):
            self.seqs[b], self.length[b] = list(self.seqs[a]), self.length[a]
            for p in self.seqs[a]:
                self.refs[p] += 1

    def trim(self, seqs, lengths):
        for s, n in zip(seqs, lengths):
            keep = -(-n // self.page)
            for p in self.seqs[s][keep:]:
                self.refs[p] -= 1
            self.seqs[s], self.length[s] = self.seqs[s][:keep], n

    def compact(self):
        live = sum(r > 0 for r in self.refs)
        holes = [i for i in range(live) if self.refs[i] == 0]
        move = [i for i in range(live, len(self.refs)) if self.refs[i] > 0]
        to = dict(zip(move, holes))
        for a, b in to.items():
            for x in self.pools + self.scales:
                x[b] = x[a]
            self.refs[b], self.refs[a] = self.refs[a], 0
        self.seqs = [[to.get(p, p) for p in s] for s in self.seqs]
        return live

    def same(self, cache):
        """State and both pools, whole."""
        assert cache.refs.tolist() == self.refs
        assert cache.length.tolist() == self.length
        assert cache.table.tolist() == [s + [-1] * (self.per - len(s)) for s in self.seqs]
        for got, want in zip((cache.k_scales, cache.v_scales), self.scales):
            assert np.array_equal(got.cpu().numpy().astype(np.float64), want, equal_nan=True)
        for got, want in zip((cache.k_pages, cache.v_pages), self.pools):
            assert same_codes(got.view(torch.uint8).cpu().numpy(), want)


def stands_for(cache, s):
    """Keys and values of sequence s as numbers of 64 bits: [length, heads, dim] each."""
    n = int(cache.length[s])
    page = cache.k_pages.shape[2]
    at = cache.table[s, :-(-n // page)].long()
    rows = []
    for pages, scales in ((cache.k_pages, cache.k_scales), (cache.v_pages, cache.v_scales)):
        if scales is None:
            x = pages[at].double()
        else:
            x = pages.view(torch.uint8)[at].view(torch.float8_e4m3fn).to(torch.float32).double()
            x = x * scales[at].double().repeat_interleave(BLOCK, 2)[..., None]
        rows.append(x.transpose(1, 2).reshape(-1, x.shape[1], x.shape[3])[:n])
    return rows


def attend8(q, k, v, scale, seen):
    """Attention of q [n, H, D] (16 bits) over k, v [m, G, D] (64 bits): out and lse, and the largest
    error of each that rounding allows.

    Codes and queries are exact in the products; one of bfloat16 loses at most 2^-39 of its row's
    largest element.  A score is a sum of D products in 32 bits, off by (D + 4) 2^-24 of their sizes,
    times a block's scale, the query's power of two and the scale of the call, 2^-22 of itself
    at most.  Its exponential carries that, and a few 2^-22 of its own.  Weights are rounded to half
    (2^-11; 2^-25 absolute, against a row sum of at least 2^8), sums add m 2^-23 at
    most, and the result is rounded once to the queries' type."""
    u = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}[q.dtype]
    tiny = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}[q.dtype]
    n, H, D = q.shape
    m, G = k.shape[:2]
    qd = q.double().view(n, G, H // G, D)
    clean = seen.any(0)
    kd, vd = (torch.where(clean[:, None, None], x, 0.0) for x in (k, v))
    s = torch.einsum("nghd,mgd->nghm", qd, kd) * scale
    size = torch.einsum("nghd,mgd->nghm", qd.abs() * (1 + 2.0 ** -24) + 2.0 ** -15 * 2.0 ** -24 * qd.abs().amax(-1, keepdim=True), kd.abs()) * abs(scale)
    hidden = ~seen[:, None, None, :]
    some = seen.any(1)[:, None, None]
    s = s.masked_fill(hidden, -math.inf)
    lse = torch.logsumexp(s, -1) if m else torch.full((n, G, H // G), -math.inf, dtype=torch.float64, device=q.device)
    p = torch.exp(s - torch.where(some, lse, 0.0)[..., None])
    out = torch.where(some[..., None], torch.einsum("nghm,mgd->nghd", p, vd), 0.0)
    off = torch.zeros_like(lse)
    top = torch.zeros((n, G, 1, D), dtype=torch.float64, device=q.device)
    if m:
        off = (size.masked_fill(hidden, 0.0) * (D + 4) * 2.0 ** -24 + s.masked_fill(hidden, 0.0).abs() * 2.0 ** -22).amax(-1)
        top = torch.where(seen[:, :, None, None].expand(-1, -1, G, D), vd.abs(), 0.0).amax(1)[:, :, None, :]
    mean = torch.einsum("nghm,mgd->nghd", p.nan_to_num(0.0), vd.abs())
    rel = 1.05 * 2.0 ** -11 + 2.0 * (off[..., None] * 1.05 + 8 * 2.0 ** -22 + m * 2.0 ** -23)
    lim = mean * rel + out.abs() * u * 1.05 + tiny + m * 2.0 ** -33 * top * 1.05 + 1e-30
    lse_lim = off * 1.05 + 2.0 ** -20 + m * 2.0 ** -23 + torch.where(some, lse, 0.0).abs() * 2.0 ** -22
    return out.reshape(n, H, D), lse.reshape(n, H), lim.reshape(n, H, D), lse_lim.reshape(n, H)

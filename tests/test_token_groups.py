"""Attention of new tokens (GPU) where a few sequences are long among very many short ones, so
that single warps have pairs of their own and the long ones' parts are joined in groups."""
import random

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from attn_util import assert_within, attend, randn  # noqa: E402
from test_cache8 import BF, DEV, E4, HF, ctx, gen, i32, offsets  # noqa: E402, F401
from window_util import attend8, near_mask, stands_for  # noqa: E402


def some_long(long, n, most, seed):
    """Lengths of n sequences of up to `most` tokens, with the long ones in pairs of neighbours, at the ends and between."""
    rng = random.Random(seed)
    lens = [rng.choice([0, 1, most, rng.randint(1, most)]) for _ in range(n)]
    at = [0, n // 2, n // 2 + 1, n - 1, n // 3, n // 3 + 1]
    for a, m in zip(at, long):
        lens[a] = m
    return lens


@pytest.mark.parametrize("long", [[200_000], [3000] * 6, [40_000, 1000, 20_003, 7, 4097, 129]])
@pytest.mark.parametrize("bits,dim,heads,kv,dtype", [(8, 64, 2, 1, BF), (8, 64, 22, 2, HF), (8, 128, 8, 1, BF), (8, 128, 12, 1, HF), (8, 96, 4, 1, BF),
                                                     (16, 64, 3, 1, HF), (16, 128, 4, 1, BF), (16, 40, 12, 1, BF)])
@pytest.mark.parametrize("window,sinks", [(None, 0), (30_000, 2000), (2 ** 31 - 1, 0)])
def test_long_among_many(ctx, long, bits, dim, heads, kv, dtype, window, sinks):  # noqa: F811
    lens = some_long(long, 2000 // kv, 150, dim + len(long))
    page, g = 32, gen(dim)
    n, per = len(lens), -(-max(lens) // page)
    c = ctx.cache(sum(-(-x // page) for x in lens) + 1, page, kv, dim, n, per, E4 if bits == 8 else dtype)
    k, v = (randn(g, (sum(lens), kv, dim), dtype) + randn(g, (1, kv, dim), dtype) for _ in range(2))
    ctx.cache_append(c, i32(range(n)), offsets(lens), k, v)
    q = randn(g, (n, heads, dim), dtype, 1.5)
    _, out, lse = ctx.cache_attention(c, None, q, need_lse=True, window=window, sinks=sinks)
    for _ in range(3):
        again = ctx.cache_attention(c, None, q, need_lse=True, window=window, sinks=sinks)
        assert torch.equal(out, again[1]) and torch.equal(lse, again[2])
    ctx.check()
    for s in [i for i, m in enumerate(lens) if m > 150] + list(range(0, n, 97)):
        kk, vv = stands_for(c, s)
        m = kk.shape[0]
        seen = near_mask(1, m, window or m, sinks, DEV) if m else torch.ones((1, 0), dtype=torch.bool, device=DEV)
        want, wl, lim, ll = (attend8 if bits == 8 else attend)(q[s:s + 1], kk, vv, dim ** -0.5, seen)
        assert_within(out[s:s + 1], want, lim, f"out of sequence {s} ({m} tokens)")
        assert_within(lse[s:s + 1], wl, ll, f"lse of sequence {s} ({m} tokens)")


def test_large_values_in_some_groups(ctx):  # noqa: F811
    """Parts whose results are held lowered, and parts whose are not, in one group and in different ones."""
    lens = some_long([200_000], 1500, 150, 1)
    g, dim = gen(2), 64
    c = ctx.cache(sum(-(-x // 16) for x in lens) + 1, 16, 1, dim, len(lens), 12_500, E4)
    k, v = randn(g, (sum(lens), 1, dim), BF), randn(g, (sum(lens), 1, dim), torch.float32).clamp(-3, 3)
    for at in (0, 50_000, 120_007, 199_990):
        v[at:at + 700] *= 2.0 ** 126
    ctx.cache_append(c, i32(range(len(lens))), offsets(lens), k, v.to(BF))
    q = randn(g, (len(lens), 4, dim), BF, 1.5)
    _, out, lse = ctx.cache_attention(c, None, q, need_lse=True)
    ctx.check()
    for s in (0, 1, 5, 1499):
        kk, vv = stands_for(c, s)
        want, wl, lim, ll = attend8(q[s:s + 1], kk, vv, dim ** -0.5, torch.ones((1, lens[s]), dtype=torch.bool, device=DEV))
        assert_within(out[s:s + 1], want, lim, f"out of sequence {s}")
        assert_within(lse[s:s + 1], wl, ll, f"lse of sequence {s}")

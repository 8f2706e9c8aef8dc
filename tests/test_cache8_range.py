"""Attention over the cache in 8 bits (GPU) at the top of the range of values that its scales
have, against 64 bits."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from attn_util import assert_within, randn  # noqa: E402
from test_cache8 import BF, DEV, E4, HF, check_attention, ctx, gen, i32, offsets  # noqa: E402, F401
from window_util import attend8, near_mask, stands_for  # noqa: E402

TOP = float(torch.finfo(BF).max)


def filled(ctx, lens, k, v, page=16):  # noqa: F811
    kv, dim = k.shape[1:]
    per = max(1, -(-max(lens) // page))
    c = ctx.cache(sum(-(-n // page) for n in lens) + 1, page, kv, dim, len(lens), per, E4)
    ctx.cache_append(c, i32(range(len(lens))), offsets(lens), k, v)
    return c



@pytest.mark.parametrize("dim,heads", [(64, 2), (128, 20), (96, 4)])
@pytest.mark.parametrize("value", [2.0 ** 112, 2.0 ** 121, -2.0 ** 125, 2.0 ** 127, TOP, -TOP])
def test_one_token(ctx, dim, heads, value):  # noqa: F811
    """A row that sees one key has its value, whatever that is."""
    k, v = torch.ones((1, 2, dim), dtype=BF, device=DEV), torch.zeros((1, 2, dim), dtype=BF, device=DEV)
    v[0, 0, ::3], v[0, 1] = value, value / 2
    c = filled(ctx, [1], k, v)
    out = ctx.cache_attention(c, None, torch.ones((1, heads, dim), dtype=BF, device=DEV))[1]
    ctx.check()
    want = stands_for(c, 0)[1].repeat_interleave(heads // 2, 1)
    assert torch.equal(out.double(), want)


@pytest.mark.parametrize("n", [2, 16, 33, 700, 5000])
@pytest.mark.parametrize("dim,heads", [(64, 2), (128, 4)])
def test_sums_of_the_largest(ctx, n, dim, heads):  # noqa: F811
    """Keys alike, each with the type's largest value: the mean is that value too."""
    k, v = torch.ones((n, 2, dim), dtype=BF, device=DEV), torch.full((n, 2, dim), TOP, dtype=BF, device=DEV)
    v[:, 1] = -TOP
    check_attention(ctx, filled(ctx, [n], k, v), torch.ones((1, heads, dim), dtype=BF, device=DEV), [0])


@pytest.mark.parametrize("size", [100, 112, 120, 126])
@pytest.mark.parametrize("dim,heads", [(64, 4), (128, 32), (48, 2)])
def test_growing_scores(ctx, size, dim, heads):  # noqa: F811
    """Scores that grow a little with every step of keys, so that sums stand above their first maximum."""
    g, n = gen(size + dim), 1500
    # (a key's score is its first element times the query's)
    k = randn(g, (n, 2, dim), BF, 2.0 ** -9)
    k[:, :, 0] = (torch.arange(n, device=DEV) / 64).to(BF)[:, None]
    v = randn(g, (n, 2, dim), torch.float32).clamp(-3, 3).mul(2.0 ** size).to(BF)
    q = randn(g, (1, heads, dim), BF, 2.0 ** -9)
    q[:, :, 0] = 1.0
    c = filled(ctx, [n], k, v)
    for scale in (1.0, 0.25, 2.0 ** -5):
        check_attention(ctx, c, q, [0], scale=scale)
        check_attention(ctx, c, q, [0], window=600, sinks=40, scale=scale)


@pytest.mark.parametrize("dim,heads,kv", [(64, 2, 2), (128, 8, 1), (128, 32, 2), (96, 4, 2)])
@pytest.mark.parametrize("at,many", [(0, 16), (39_984, 16), (20_001, 1), (10_000, 9_000), (0, 40_000)])
def test_some_are_large(ctx, dim, heads, kv, at, many):  # noqa: F811
    """Many small values and a run of large ones, in parts of a sequence that are joined; a
    log-sum-exp that does not depend on values."""
    g, lens = gen(at + dim), [40_000, 300]
    n = sum(lens)
    k = randn(g, (n, kv, dim), BF)
    v = randn(g, (n, kv, dim), torch.float32).clamp(-3, 3)
    plain = filled(ctx, lens, k, v.to(BF), 64)
    v[at:at + many] *= 2.0 ** 126
    c = filled(ctx, lens, k, v.to(BF), 64)
    q = randn(g, (2, heads, dim), BF, 1.5)
    out, lse = check_attention(ctx, c, q, [0, 1])
    want = ctx.cache_attention(plain, None, q, need_lse=True)
    assert torch.equal(lse, want[2]) and torch.equal(out[1], want[1][1])
    check_attention(ctx, c, q, [0, 1], window=15_000, sinks=100)


@pytest.mark.parametrize("dim", [64, 128, 80])
@pytest.mark.parametrize("window,sinks", [(None, 0), (100, 20)])
def test_many_sequences(ctx, dim, window, sinks):  # noqa: F811
    """Pairs of a warp's own, one after another: large values of one have no part in the next."""
    g, kv, heads = gen(dim), 4, 8
    lens = [1 + 37 * i % 300 for i in range(600)] + [9000]
    n = sum(lens)
    k, v = randn(g, (n, kv, dim), BF), randn(g, (n, kv, dim), torch.float32).clamp(-3, 3)
    plain = filled(ctx, lens, k, v.to(BF), 32)
    ends = offsets(lens).tolist()
    odd = torch.zeros(n, dtype=torch.bool, device=DEV)
    for s in range(0, len(lens), 3):
        odd[(ends[s] + ends[s + 1]) // 2:ends[s + 1]] = True
    v = torch.where(odd[:, None, None], v * 2.0 ** 126, v)
    c = filled(ctx, lens, k, v.to(BF), 32)
    q = randn(g, (len(lens), heads, dim), BF, 1.5)
    _, out, lse = ctx.cache_attention(c, None, q, need_lse=True, window=window, sinks=sinks)
    _, want, want_lse = ctx.cache_attention(plain, None, q, need_lse=True, window=window, sinks=sinks)
    ctx.check()
    assert torch.equal(lse, want_lse)
    calm = torch.tensor([i % 3 != 0 for i in range(len(lens))], device=DEV)
    assert torch.equal(out[calm], want[calm])
    for s in list(range(0, 90, 3)) + [600]:
        kk, vv = stands_for(c, s)
        m = kk.shape[0]
        exact, _, lim, _ = attend8(q[s:s + 1], kk, vv, dim ** -0.5, near_mask(1, m, window or m, sinks, DEV))
        assert_within(out[s:s + 1], exact, lim, f"out of sequence {s} ({m} tokens)")


def test_scales_of_others(ctx):  # noqa: F811
    """Scales that the caller wrote, of either sign and no powers of two, for rows of half."""
    g = gen(3)
    k, v = (randn(g, (300, 2, 64), HF) for _ in range(2))
    c = filled(ctx, [300], k, v)
    c.v_scales.mul_(torch.tensor([1.0, -3e37], device=DEV)[torch.arange(c.v_scales.numel(), device=DEV).view_as(c.v_scales) % 2])
    q = randn(g, (1, 4, 64), BF, 1.5)
    check_attention(ctx, c, q, [0])
    c.v_scales[2, 0, 0] = math.nan
    out = ctx.cache_attention(c, None, q)[1]
    assert out[0, :2].isnan().all() and out[0, 2:].isfinite().all()


@pytest.mark.parametrize("dim,heads", [(64, 4), (128, 4)])
@pytest.mark.parametrize("bits", [10, 24, 30, 32, 33, 34, 40, 70])
def test_small_weights_of_large_values(ctx, dim, heads, bits):  # noqa: F811
    """A block of values 2^60 times the others' at weights 2^-bits of the largest: a weight is off by 2^-11 of
    itself, or 2^-33 of the largest, whatever its value; one above 2^-32 of it still counts."""
    k, v = torch.zeros((48, 1, dim), dtype=BF, device=DEV), torch.ones((48, 1, dim), dtype=BF, device=DEV)
    k[:16, 0, 0], v[16:32, 0, ::2] = 1.0, 2.0 ** 60
    # scores 0 and -bits, in powers of two
    q = torch.zeros((1, heads, dim), dtype=BF, device=DEV)
    q[:, :, 0] = 1.0
    scale = bits * math.log(2.0)
    c = filled(ctx, [48], k, v)
    out, _ = check_attention(ctx, c, q, [0], scale=scale)
    # (16 keys with weight 1, 32 with 2^-bits, 16 of which have the large values)
    want = 2.0 ** (60 - bits) + 1.0
    if bits < 33:
        assert ((out[:, :, ::2].double() / want - 1).abs() < 2.0 ** -7 + 2.0 ** (bits - 33)).all()
    assert ((out[:, :, 1::2].double() - 1.0).abs() < 2.0 ** -7).all()


@pytest.mark.parametrize("dim,heads", [(64, 4), (128, 12), (48, 2)])
@pytest.mark.parametrize("small", [-98, -105, -112, -118, -124])
@pytest.mark.parametrize("bits", [0, 6, 13])
def test_small_queries_of_large_keys(ctx, dim, heads, small, bits):  # noqa: F811
    """Queries near bfloat16's least numbers, keys large enough that their scores count, and a small scale."""
    g, n = gen(-small + dim), 300
    k = randn(g, (n, 2, dim), torch.float32).clamp(-3, 3).mul(2.0 ** min(126, -small + bits)).to(BF)
    v = randn(g, (n, 2, dim), BF)
    q = randn(g, (1, heads, dim), torch.float32).mul(2.0 ** small).to(BF)
    check_attention(ctx, filled(ctx, [n], k, v), q, [0], scale=2.0 ** -bits)


@pytest.mark.parametrize("dim,heads", [(64, 2), (128, 20), (80, 2)])
@pytest.mark.parametrize("size", [1.0, -1.0])
def test_products_of_zero(ctx, dim, heads, size):  # noqa: F811
    """Scales whose product with a query's size leaves 32 bits: a key whose products are all zero has the score 0."""
    n = 40
    g = gen(dim)
    k, v = torch.zeros((n, 2, dim), dtype=BF, device=DEV), randn(g, (n, 2, dim), BF)
    k[:, :, 1] = 2.0 ** 100                             # (queries have zeros there)
    k[7, :, 0], k[23, :, 0] = -size * 2.0 ** 100, -size * 2.0 ** 99
    q = torch.zeros((1, heads, dim), dtype=BF, device=DEV)
    q[:, :, 0] = size * 2.0 ** 100
    c = filled(ctx, [n], k, v)
    _, out, lse = ctx.cache_attention(c, None, q, need_lse=True)
    ctx.check()
    rest = [i for i in range(n) if i not in (7, 23)]
    want = stands_for(c, 0)[1][rest].mean(0).repeat_interleave(heads // 2, 0)
    assert ((out[0].double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -10 * v.abs().max()).all()
    assert ((lse.double() - math.log(len(rest))).abs() <= 2.0 ** -18).all()

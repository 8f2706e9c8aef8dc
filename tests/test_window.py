"""Attention through a sliding window with sinks (GPU), over prompts and over the paged
cache, against its definition in 64 bits."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from attn_util import assert_within, attend, randn  # noqa: E402
from window_util import near_mask  # noqa: E402

DEV = "cuda:0"
BF, HF = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def ctx():
    import paper_2609_11938_gb300 as opa
    with opa.Context(0) as c:
        yield c


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def offsets(lens):
    return i32([0] + [sum(lens[:i + 1]) for i in range(len(lens))])


def check_prompt(ctx, q, k, v, lq, lk, window, sinks, scale=None, **kw):
    _, out, lse = ctx.attention(q, k, v, offsets(lq), offsets(lk), scale=scale, need_lse=True, window=window, sinks=sinks, **kw)
    ctx.check()
    a = b = 0
    for i, (n, m) in enumerate(zip(lq, lk)):
        seen = near_mask(n, m, window, sinks, DEV)
        want, wl, lim, ll = attend(q[a:a + n], k[b:b + m], v[b:b + m], q.shape[2] ** -0.5 if scale is None else scale, seen)
        assert_within(out[a:a + n], want, lim, f"out of sequence {i} ({n} queries, {m} keys)")
        assert_within(lse[a:a + n], wl, ll, f"lse of sequence {i} ({n} queries, {m} keys)")
        a, b = a + n, b + m
    return out, lse


@pytest.mark.parametrize("dtype,dim,heads,kv", [(BF, 64, 3, 3), (HF, 128, 4, 1), (BF, 96, 10, 2), (HF, 8, 2, 2)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (7, 4), (64, 0), (128, 130), (129, 127), (300, 5), (2 ** 31 - 1, 3), (40, 2 ** 31 - 1)])
@pytest.mark.parametrize("lens", [[1], [2, 1, 3], [127, 128, 129], [255, 0, 257, 511], [900, 1]])
def test_prompts(ctx, dtype, dim, heads, kv, window, sinks, lens):
    g = gen(sum(lens) + dim + window % 1000)
    t = sum(lens)
    q, k, v = randn(g, (t, heads, dim), dtype, 1.5), randn(g, (t, kv, dim), dtype), randn(g, (t, kv, dim), dtype)
    check_prompt(ctx, q, k, v, lens, lens, window, sinks)


@pytest.mark.parametrize("window,sinks", [(1, 0), (100, 3), (128, 0), (1000, 200), (4096, 1)])
@pytest.mark.parametrize("lq,lk", [([1, 5, 130], [700, 5, 1300]), ([64] * 3, [3001, 64, 65]), ([300, 20], [120, 0])])
@pytest.mark.parametrize("heads,kv,dim", [(20, 4, 96), (8, 1, 64), (2, 2, 128)])
def test_keys_before_the_queries(ctx, window, sinks, lq, lk, heads, kv, dim):
    """Pieces of prompts; queries before the first key see nothing."""
    g = gen(window + sum(lk))
    q = randn(g, (sum(lq), heads, dim), BF, 1.5)
    k, v = (randn(g, (sum(lk), kv, dim), BF) for _ in range(2))
    check_prompt(ctx, q, k, v, lq, lk, window, sinks)


@pytest.mark.parametrize("window,sinks,n,m,heads,kv", [(6000, 4, 1, 20000, 8, 8), (9000, 0, 70, 20003, 8, 2), (15000, 600, 300, 15100, 4, 4),
                                                       (20000, 4, 3, 20000, 16, 2)])
def test_few_queries_are_cut(ctx, window, sinks, n, m, heads, kv):
    """Few queries over a wide window: its tiles are shared out, and parts joined."""
    g = gen(n)
    q = randn(g, (n, heads, 128), BF, 1.5)
    k, v = (randn(g, (m, kv, 128), BF) for _ in range(2))
    a, b = (check_prompt(ctx, q, k, v, [n], [m], window, sinks) for _ in range(2))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_many_sequences(ctx):
    """More sequences than a warp has lanes, most of them short."""
    g = gen(5)
    lens = [int(x) for x in torch.randint(0, 90, (150,), generator=g, device=DEV)] + [700]
    q, k, v = randn(g, (sum(lens), 6, 64), BF, 1.5), randn(g, (sum(lens), 2, 64), BF), randn(g, (sum(lens), 2, 64), BF)
    check_prompt(ctx, q, k, v, lens, lens, 33, 2)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("window,sinks", [(20, 0), (150, 3), (1, 0)])
@pytest.mark.parametrize("bad", [math.inf, math.nan])
def test_values_out_of_sight(ctx, dtype, window, sinks, bad):
    """Keys and values that a row does not see have no influence on it, whatever they hold."""
    g = gen(3)
    n, at = 600, 290
    q, k, v = randn(g, (n, 2, 64), dtype, 1.5), randn(g, (n, 2, 64), dtype), randn(g, (n, 2, 64), dtype)
    _, want, wl = ctx.attention(q, k, v, offsets([n]), window=window, sinks=sinks, need_lse=True)
    k2, v2 = k.clone(), v.clone()
    k2[at], v2[at] = bad, -bad
    _, out, lse = ctx.attention(q, k2, v2, offsets([n]), window=window, sinks=sinks, need_lse=True)
    ctx.check()
    free = torch.ones(n, dtype=torch.bool, device=DEV)
    free[at:at + window] = False
    assert torch.isfinite(out[free]).all() and not torch.isfinite(out[~free]).any()
    # (the tile's products are made in another order there)
    lim = attend(q, k, v, 64 ** -0.5, near_mask(n, n, window, sinks, DEV))[2]
    assert ((out.double() - want.double()).abs()[free] <= 2 * lim[free]).all()
    assert torch.equal(lse[free], wl[free])


def test_wide_window_is_none(ctx):
    g = gen(9)
    n = 500
    q, k, v = randn(g, (n, 4, 64), HF, 1.5), randn(g, (n, 2, 64), HF), randn(g, (n, 2, 64), HF)
    a = ctx.attention(q, k, v, offsets([200, 300]), need_lse=True)
    for window, sinks in ((300, 0), (2 ** 31 - 1, 0), (1, 300)):
        b = ctx.attention(q, k, v, offsets([200, 300]), need_lse=True, window=window, sinks=sinks)
        assert torch.equal(a[1], b[1]) and torch.equal(a[2], b[2])


def test_strides_and_scale(ctx):
    g = gen(11)
    n = 333
    big = randn(g, (n, 9, 3 * 64), BF)
    q, k, v = big[:, :8, :64], big[:, 1:3, 64:128], big[:, 3:4, 128:].expand(n, 2, 64)
    out = torch.empty((n, 12, 64), dtype=BF, device=DEV)[:, 2:10]
    got, _ = check_prompt(ctx, q, k, v, [300, 33], [300, 33], 50, 2, scale=-0.3, out=out)
    assert got is out


# ---------------------------------------------------------------- tokens over the cache
def filled(ctx, lens, page, kv, dim, dtype, seed, spare=0):
    g = gen(seed)
    per = max(1, -(-(max(lens) + spare) // page))
    c = ctx.cache(per * len(lens) + 3, page, kv, dim, len(lens), per, dtype)
    k, v = (randn(g, (sum(lens), kv, dim), dtype) for _ in range(2))
    ctx.cache_append(c, i32(range(len(lens))), offsets(lens), k, v)
    # pages in no order
    to = torch.randperm(c.refs.numel(), generator=g, device=DEV)
    for x in ("k_pages", "v_pages", "refs"):
        old = getattr(c, x).clone()
        getattr(c, x)[to] = old
    c.table.copy_(torch.where(c.table >= 0, to[c.table.clamp(min=0).long()].int(), c.table))
    return c, k, v, g


def check_token(ctx, c, k, v, lens, q, seqs, window, sinks):
    _, out, lse = ctx.cache_attention(c, i32(seqs), q, need_lse=True, window=window, sinks=sinks)
    ctx.check()
    starts = [sum(lens[:i]) for i in range(len(lens))]
    for i, s in enumerate(seqs):
        a, n = starts[s], lens[s]
        seen = near_mask(1, n, window, sinks, DEV) if n else torch.ones((1, 0), dtype=torch.bool, device=DEV)
        want, wl, lim, ll = attend(q[i:i + 1], k[a:a + n], v[a:a + n], q.shape[2] ** -0.5, seen)
        assert_within(out[i:i + 1], want, lim, f"out of sequence {s} ({n} tokens)")
        assert_within(lse[i:i + 1], wl, ll, f"lse of sequence {s} ({n} tokens)")


@pytest.mark.parametrize("dtype,dim,heads,kv,page", [(BF, 64, 12, 12, 16), (HF, 128, 8, 2, 32), (BF, 128, 24, 2, 64), (HF, 64, 11, 1, 16), (BF, 40, 3, 3, 128)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (16, 1), (100, 4), (128, 200), (1000, 0), (2 ** 31 - 1, 4), (5, 2 ** 31 - 1)])
def test_tokens(ctx, dtype, dim, heads, kv, page, window, sinks):
    lens = [1, 0, 15, 16, 17, 128, 129, 700, 1025, 3000]
    c, k, v, g = filled(ctx, lens, page, kv, dim, dtype, window % 1000 + dim)
    seqs = list(range(len(lens))) + [7, 9, 9]
    check_token(ctx, c, k, v, lens, randn(g, (len(seqs), heads, dim), dtype, 1.5), seqs, window, sinks)


@pytest.mark.parametrize("dim,heads,dtype", [(64, 4, BF), (40, 48, HF), (128, 8, HF), (96, 40, BF)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (100, 20), (3000, 1)])
def test_many_pairs(ctx, dim, heads, dtype, window, sinks):
    """So many sequences and key heads that each warp has its own, with some among them that many warps share."""
    g = gen(dim)
    lens = torch.randint(0, 300, (490,), generator=g, device=DEV).tolist() + [9000, 0, 1, 3001, 700]
    c, k, v, g = filled(ctx, lens, 32, 4, dim, dtype, dim)
    seqs = torch.randperm(len(lens), generator=g, device=DEV).tolist()
    q = randn(g, (len(lens), heads, dim), dtype, 1.5)
    a, b = (ctx.cache_attention(c, i32(seqs), q, need_lse=True, window=window, sinks=sinks) for _ in range(2))
    ctx.check()
    assert torch.equal(a[1], b[1]) and torch.equal(a[2], b[2])
    starts = [sum(lens[:i]) for i in range(len(lens))]
    for i, s in enumerate(seqs):
        at, n = starts[s], lens[s]
        if n < 600 and i % 9:
            continue
        seen = near_mask(1, n, window, sinks, DEV) if n else torch.ones((1, 0), dtype=torch.bool, device=DEV)
        want, wl, lim, ll = attend(q[i:i + 1], k[at:at + n], v[at:at + n], dim ** -0.5, seen)
        assert_within(a[1][i:i + 1], want, lim, f"out of sequence {s} ({n} tokens)")
        assert_within(a[2][i:i + 1], wl, ll, f"lse of sequence {s} ({n} tokens)")


@pytest.mark.parametrize("window,sinks", [(20_000, 4), (30_000, 9000), (64, 0)])
def test_long_contexts(ctx, window, sinks):
    """Windows of many blocks' runs, and one that is little of what there is."""
    lens = [40_000, 33]
    c, k, v, g = filled(ctx, lens, 64, 2, 128, BF, 3)
    q = randn(g, (2, 8, 128), BF, 1.5)
    check_token(ctx, c, k, v, lens, q, [0, 1], window, sinks)
    a, b = (ctx.cache_attention(c, i32([0, 1]), q, window=window, sinks=sinks)[1] for _ in range(2))
    assert torch.equal(a, b)


@pytest.mark.parametrize("bad", [math.inf, math.nan])
def test_tokens_out_of_sight(ctx, bad):
    """What lies before the window, and pages that are none there, have no influence."""
    n, window, sinks = 1000, 100, 20
    c, k, v, g = filled(ctx, [n], 16, 2, 64, BF, 4)
    q = randn(g, (1, 4, 64), BF, 1.5)
    want = ctx.cache_attention(c, i32([0]), q, window=window, sinks=sinks, need_lse=True)
    for t in range(sinks, n - window):
        p = int(c.table[0, t // 16])
        c.k_pages[p, :, t % 16] = bad
        c.v_pages[p, :, t % 16] = bad
    c.table[0, 2:(n - window) // 16] = -1
    got = ctx.cache_attention(c, i32([0]), q, window=window, sinks=sinks, need_lse=True)
    ctx.check()
    assert torch.equal(got[1], want[1]) and torch.equal(got[2], want[2])


def test_page_out_of_range(ctx):
    import paper_2609_11938_gb300 as opa
    c, _, _, g = filled(ctx, [300], 16, 1, 64, BF, 6)
    q = randn(g, (1, 2, 64), BF)
    c.table[0, 18] = 10 ** 6
    ctx.cache_attention(c, i32([0]), q, window=5)
    with pytest.raises(opa.OpattrError, match="invalid argument"):
        ctx.check()
    ctx.check()


def test_other_stream(ctx):
    """A call on another stream than the context's, of inputs that are still being made there."""
    s = torch.cuda.Stream()
    c, k, v, g = filled(ctx, [500], 16, 2, 64, BF, 8)
    q = randn(g, (1, 4, 64), BF, 1.5)
    want = ctx.cache_attention(c, i32([0]), q, window=77, sinks=1)[1]
    prompt = ctx.attention(q.expand(1, 4, 64), k[:1], v[:1], offsets([1]), window=3)[1]
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(2_000_000)
        q2 = q * 1
        got = ctx.cache_attention(c, None, q2, window=77, sinks=1)[1].clone()
        p2 = ctx.attention(q2, k[:1], v[:1], window=3)[1].clone()
    s.synchronize()
    assert torch.equal(got, want) and torch.equal(p2, prompt)
    ctx.check()

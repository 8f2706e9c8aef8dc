"""Windows and caches in 8 bits at the largest numbers of tokens (GPU): places a step or a
tile past the last one pass 32 bits; and waits of windowed prompts that run out."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from attn_util import attend, randn  # noqa: E402
from window_util import near_mask  # noqa: E402

DEV = "cuda:0"
BF, E4 = torch.bfloat16, torch.float8_e4m3fn
MOST = 2 ** 31 - 1


@pytest.fixture(scope="module")
def opa():
    import paper_2609_11938_gb300 as opa
    return opa


@pytest.fixture(scope="module")
def ctx(opa):
    with opa.Context(0) as c:
        yield c


def i32(*x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


KINDS = [(False, 8), (False, 72), (True, 16), (True, 64), (True, 128)]        # 8 bits, and the width
VIEWS = [(None, 0), (1000, 0), (1000, 1000), (5, 1), (MOST, MOST), (1, MOST), (MOST // 2, 0)]


@pytest.mark.parametrize("page,short", [(1024, 0), (1024, 1), (16, 0), (16, 17)])
@pytest.mark.parametrize("eight,dim,window,sinks", [k + v for k in KINDS for v in VIEWS if k[0] or v[0]])
def test_token_longest(opa, ctx, eight, dim, page, short, window, sinks):
    """A sequence as long as a table can say, all of whose pages but the last are the same one.  The
    first head sees all keys alike, half with a value of 1 and half of 3; the second nothing but the
    last key."""
    per = MOST // page
    length = per * page - short
    k, v = (torch.zeros((2, 1, page, dim), device=DEV) for _ in range(2))
    v[:, :, ::2], v[:, :, 1::2] = 1.0, 3.0
    table = torch.zeros((1, per), dtype=torch.int32, device=DEV)
    table[0, (length - 1) // page:] = 1
    at = (length - 1) % page
    k[1, 0, at, 0], v[1, 0, at] = 192.0, 5.0
    scales = [torch.ones((2, 1, page // 16), device=DEV) for _ in range(2)] if eight else []
    c = opa.KVCache(k.to(E4 if eight else BF), v.to(E4 if eight else BF), table, i32(length), i32(1, 1), i32(0), *scales)
    q = torch.zeros((1, 2, dim), dtype=BF, device=DEV)
    q[0, 1, 0] = 1.0
    _, out, lse = ctx.cache_attention(c, None, q, scale=1.0, need_lse=True, window=window, sinks=sinks)
    ctx.check()
    seen = length if window is None else min(length, window + min(sinks, length - min(window, length)))
    # the last key's value is 5, and of the others there are as many of 1 as of 3, or one more
    first = [(i, 1 if i % 2 == 0 else 3) for i in range(min(sinks, 2))]
    assert (out[0, 1] == 5).all() and abs(float(lse[0, 1]) - 192) < 1e-4
    if seen > 10:
        assert abs(float(out[0, 0, 0]) - 2) <= 2 * 2 ** -8 + 4 / seen
    elif seen == 6:                                      # the first key and the last five
        near = [(3 if (length - 5 + i) % 2 else 1) for i in range(4)] + [5]
        assert abs(float(out[0, 0, 0]) - (first[0][1] + sum(near)) / 6) <= 4 * 2 ** -8
    assert abs(float(lse[0, 0]) - math.log(seen)) < 1e-4


@pytest.mark.parametrize("window,sinks", [(1000, 0), (3001, 1000), (64, 1), (MOST, MOST), (1, MOST), (MOST - 200, 100), (MOST - 16, 0)])
def test_prompt_most_keys(ctx, window, sinks):
    n = MOST
    kv = torch.zeros((n, 1, 8), dtype=BF, device=DEV)
    kv[::2, 0, 1], kv[1::2, 0, 1] = 1.0, 3.0
    kv[-1, 0, 0], kv[-1, 0, 1] = 200.0, 5.0
    q = torch.zeros((1, 2, 8), dtype=BF, device=DEV)
    q[0, 1, 0] = 1.0
    _, out, lse = ctx.attention(q, kv, kv, i32(0, 1), i32(0, n), scale=1.0, need_lse=True, window=window, sinks=sinks)
    ctx.check()
    seen = min(n, window + min(sinks, n - min(window, n)))
    assert out[0, 1].tolist() == [200.0, 5.0] + [0.0] * 6 and abs(float(lse[0, 1]) - 200) < 1e-4
    assert abs(float(out[0, 0, 1]) - 2) <= 2 * 2 ** -8 + 4 / seen and abs(float(lse[0, 0]) - math.log(seen)) < 1e-4


@pytest.mark.parametrize("window,sinks", [(2, 1), (MOST, 0)])
def test_prompt_most_queries(ctx, window, sinks):
    """Queries before the one key see nothing; the last one sees it."""
    n = MOST
    q = torch.zeros((n, 1, 8), dtype=BF, device=DEV)
    k = torch.full((1, 1, 8), 3.0, dtype=BF, device=DEV)
    out = torch.full_like(q, 7.0)
    ctx.attention(q, k, k, i32(0, n), i32(0, 1), out=out, window=window, sinks=sinks)
    ctx.check()
    assert (out[-1] == 3).all()
    assert all(bool((x == 0).all()) for x in out[:-1].split(1 << 27))


def inputs(queries, keys, heads, kv, dim, dtype):
    g = torch.Generator(device=DEV)
    g.manual_seed(queries + keys)
    q = randn(g, (queries, heads, dim), dtype)
    k, v = (randn(g, (keys, kv, dim), dtype) for _ in range(2))
    return q, k, v, i32(0, queries), i32(0, keys)


@pytest.mark.parametrize("silent", [1, 2, 5, 9, -1])
@pytest.mark.parametrize("queries,keys,heads,kv,dim,dtype,window,sinks,tiles", [(1000, 1000, 8, 2, 128, BF, 200, 4, 6), (900, 1300, 3, 3, 64, torch.float16, 500, 130, 12),
                                                                                (20, 9000, 8, 2, 64, BF, 8000, 20, 10)])
def test_waits_run_out(opa, monkeypatch, queries, keys, heads, kv, dim, dtype, window, sinks, tiles, silent):
    """Copies that end before a block's N-th tile; for -1 a warp that does not come where parts are
    joined, which only calls that cut keys do.  `tiles`: copies that some block has at least, and in the first
    case all have at most (an item of 64 tokens: 16 + 200 + 63 keys, of which the tiles are copied for
    keys and for values; fewer items than SMs), so that the ninth is never begun there."""
    args, kw = inputs(queries, keys, heads, kv, dim, dtype), dict(window=window, sinks=sinks)
    with opa.Context(0) as ctx:
        want = ctx.attention(*args, **kw)[1]
        ctx.check()
    monkeypatch.setenv("OPATTR_FAULT", f"prompt:{silent}")
    with opa.Context(0) as ctx:
        first = ctx.attention(*args, **kw)[1]
        monkeypatch.delenv("OPATTR_FAULT")
        if (silent < 0 and queries > 500) or silent > tiles:
            ctx.check()
            assert torch.equal(first, want)
        else:
            ctx.attention(*args, **kw)                   # begins nothing: what is left behind is not used
            with pytest.raises(opa.OpattrError) as e:
                ctx.check()
            assert e.value.status == opa.E_TIMEOUT
        for _ in range(2):
            assert torch.equal(ctx.attention(*args, **kw)[1], want)
            ctx.check()


@pytest.mark.parametrize("bad", [math.inf, math.nan])
@pytest.mark.parametrize("sinks", [0, 4, 130])
def test_out_of_sight_where_keys_are_cut(ctx, bad, sinks):
    """Few queries over a wide window, whose tiles are shared out: what lies before it, between the
    sinks and it, and behind the keys, has no influence."""
    n, m, window = 20, 12_000, 9_000
    q, k, v, qo, _ = inputs(n, m + 300, 8, 2, 128, BF)
    ko = i32(0, 0, m)                                    # a sequence without keys before it, rows of nobody behind
    hidden = torch.ones(m + 300, dtype=torch.bool, device=DEV)
    seen = near_mask(n, m, window, sinks, DEV)
    hidden[:m] = ~seen.any(0)
    k, v = k[:m], v[:m]
    clean = ctx.attention(q, k, v, i32(0, 0, n), ko, window=window, sinks=sinks)[1]
    k2, v2 = k.clone(), v.clone()
    k2[hidden[:m]], v2[hidden[:m]] = bad, bad
    # and one that the last queries alone do not see
    edge = m - n - window + 1
    assert seen[0, edge] and not seen[-1, edge]
    got = ctx.attention(q, k2, v2, i32(0, 0, n), ko, window=window, sinks=sinks)[1]
    ctx.check()
    lim = attend(q, k, v, 128 ** -0.5, seen)[2]
    assert ((got.double() - clean.double()).abs() <= 2 * lim).all()
    k2[edge], v2[edge] = bad, -bad
    got = ctx.attention(q, k2, v2, i32(0, 0, n), ko, window=window, sinks=sinks)[1]
    ctx.check()
    blind = ~seen[:, edge]
    assert not torch.isfinite(got[~blind]).any()
    assert ((got.double() - clean.double()).abs() <= 2 * lim)[blind].all()

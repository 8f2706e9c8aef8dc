"""Attention over many keys, half and bfloat16 (GPU), within bounds that tell a result that is
missing, turned or short of a tile of keys (test_attn_bound.py) from a right one."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from attn_bound import bound, misses  # noqa: E402
from attn_util import causal_mask, randn  # noqa: E402

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


def offsets(lens):
    return torch.tensor([0] + list(torch.tensor(lens).cumsum(0)), dtype=torch.int32, device=DEV)


def check(got, q, k, v, seen, what):
    wrong = misses(got, *bound(q, k, v, q.shape[2] ** -0.5, seen))
    assert wrong is None, f"{what}: {wrong}"


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dim,heads,kv,lq,lk", [
    (64, 3, 1, [1], [20_000]), (64, 4, 2, [300, 1, 40], [9001, 30, 5000]), (128, 4, 2, [2, 257], [30_001, 4999]),
    (128, 6, 3, [200], [4100]), (96, 4, 1, [129, 60], [9000, 1500]), (40, 2, 2, [7] * 30, [3000 + 97 * i for i in range(30)]),
    (128, 2, 1, [1500], [1500]), (64, 8, 8, [700, 900], [700, 900])])
def test_prompt(ctx, dtype, causal, dim, heads, kv, lq, lk):
    g = gen(sum(lk) + dim)
    q = randn(g, (sum(lq), heads, dim), dtype)
    k, v = (randn(g, (sum(lk), kv, dim), dtype) for _ in range(2))
    out = ctx.attention(q, k, v, offsets(lq), offsets(lk), causal=causal)[1]
    ctx.check()
    a = b = 0
    for i, (n, m) in enumerate(zip(lq, lk)):
        seen = causal_mask(n, m, DEV) if causal else torch.ones((n, m), dtype=torch.bool, device=DEV)
        for at in range(0, n, 256):
            rows = slice(a + at, a + min(at + 256, n))
            check(out[rows], q[rows], k[b:b + m], v[b:b + m], seen[at:at + 256], f"sequence {i}, queries from {at}")
        a, b = a + n, b + m


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dim,heads,kv,page,lens", [
    (64, 6, 2, 16, [1500, 700]), (128, 8, 1, 32, [9000]), (128, 40, 8, 64, [40_001, 3000]), (80, 7, 1, 16, [3000, 100, 12_000]),
    (64, 34, 2, 128, [30_000, 5000, 333])])
def test_token(ctx, dtype, dim, heads, kv, page, lens):
    g = gen(sum(lens) + dim)
    c = ctx.cache(sum(-(-n // page) for n in lens), page, kv, dim, len(lens), -(-max(lens) // page), dtype)
    k, v = (randn(g, (sum(lens), kv, dim), dtype) for _ in range(2))
    ctx.cache_append(c, torch.arange(len(lens), dtype=torch.int32, device=DEV), offsets(lens), k, v)
    q = randn(g, (len(lens), heads, dim), dtype)
    out = ctx.cache_attention(c, None, q)[1]
    ctx.check()
    a = 0
    for i, n in enumerate(lens):
        check(out[i:i + 1], q[i:i + 1], k[a:a + n], v[a:a + n], torch.ones((1, n), dtype=torch.bool, device=DEV), f"sequence {i}")
        a += n


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dim,n,at", [(64, 40, 7), (128, 3000, 2999), (64, 9000, 0)])
def test_token_seen_infinite_value(ctx, dtype, dim, n, at):
    """An infinite value that is seen is the result, in its element alone."""
    g = gen(n)
    c = ctx.cache(-(-n // 16), 16, 1, dim, 1, -(-n // 16), dtype)
    k, v = (randn(g, (n, 1, dim), dtype) for _ in range(2))
    k[:] = 0.0
    v[at, 0, 5] = float("inf")
    ctx.cache_append(c, torch.zeros(1, dtype=torch.int32, device=DEV), offsets([n]), k, v)
    out = ctx.cache_attention(c, None, randn(g, (1, 4, dim), dtype))[1]
    ctx.check()
    assert bool((out[0, :, 5] == float("inf")).all()) and int(torch.isfinite(out).sum()) == 4 * (dim - 1)

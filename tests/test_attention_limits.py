"""The largest numbers of tokens that the attention operators take (GPU): places
a step or a tile past the last one pass 32 bits."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

DEV = "cuda:0"
BF = torch.bfloat16


@pytest.fixture(scope="module")
def ctx():
    import paper_2609_11938_gb300 as opa
    with opa.Context(0) as c:
        yield c


def i32(*x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("dim", [8, 72])
@pytest.mark.parametrize("page,short", [(1024, 0), (1024, 1), (16, 0), (16, 15), (16, 17), (16, 4000)])
def test_token_longest(ctx, dim, page, short):
    """A sequence as long as a table can say, all of whose pages but the last are the same one.
    The first head sees all keys alike, half with a value of 1 and half of 3; the second
    nothing but the last key."""
    import paper_2609_11938_gb300 as opa
    per = (2 ** 31 - 1) // page
    length = per * page - short
    k, v = (torch.zeros((2, 1, page, dim), dtype=BF, device=DEV) for _ in range(2))
    v[:, :, ::2], v[:, :, 1::2] = 1.0, 3.0
    table = torch.zeros((1, per), dtype=torch.int32, device=DEV)
    table[0, (length - 1) // page:] = 1
    at = (length - 1) % page
    k[1, 0, at, 0], v[1, 0, at] = 200.0, 5.0
    c = opa.KVCache(k, v, table, i32(length), i32(1, 1), i32(0))
    q = torch.zeros((1, 2, dim), dtype=BF, device=DEV)
    q[0, 1, 0] = 1.0
    _, out, lse = ctx.cache_attention(c, None, q, scale=1.0, need_lse=True)
    ctx.check()
    assert (out[0, 0] == 2).all() and (out[0, 1] == 5).all()
    assert abs(float(lse[0, 0]) - math.log(length)) < 1e-4 and abs(float(lse[0, 1]) - 200) < 1e-4


@pytest.mark.parametrize("causal", [True, False])
def test_prompt_most_keys(ctx, causal):
    n = 2 ** 31 - 1
    kv = torch.zeros((n, 1, 8), dtype=BF, device=DEV)
    kv[::2, 0, 1], kv[1::2, 0, 1] = 1.0, 3.0
    kv[-1, 0, 0], kv[-1, 0, 1] = 200.0, 5.0
    q = torch.zeros((1, 2, 8), dtype=BF, device=DEV)
    q[0, 1, 0] = 1.0
    _, out, lse = ctx.attention(q, kv, kv, i32(0, 1), i32(0, n), causal=causal, scale=1.0, need_lse=True)
    ctx.check()
    assert out[0, 0].tolist()[1:] == [2.0] + [0.0] * 6 and out[0, 1].tolist() == [200.0, 5.0] + [0.0] * 6
    assert abs(float(lse[0, 0]) - math.log(n)) < 1e-4 and abs(float(lse[0, 1]) - 200) < 1e-4


@pytest.mark.parametrize("causal", [True, False])
def test_prompt_most_queries(ctx, causal):
    n = 2 ** 31 - 1
    q = torch.zeros((n, 1, 8), dtype=BF, device=DEV)
    k = torch.full((1, 1, 8), 3.0, dtype=BF, device=DEV)
    out = torch.full_like(q, 7.0)
    ctx.attention(q, k, k, i32(0, n), i32(0, 1), causal=causal, out=out)
    ctx.check()
    assert (out[-1] == 3).all()                          # the last query sees the key, with a mask as well
    rest = 0 if causal else 3
    assert all(bool((x == rest).all()) for x in out[:-1].split(1 << 27))

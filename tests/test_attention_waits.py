"""The prompt kernel's waits run out (GPU): a part of every block falls silent
(OPATTR_FAULT=prompt:N, the first prompt call of a context), the others give up after
a short limit, the call's end is told by opattr_check, and the context goes on."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from attn_util import randn  # noqa: E402

DEV = "cuda:0"


@pytest.fixture(scope="module")
def opa():
    import paper_2609_11938_gb300 as opa
    return opa


def inputs(queries, keys, heads, kv, dim, dtype):
    g = torch.Generator(device=DEV)
    g.manual_seed(queries + keys)
    q = randn(g, (queries, heads, dim), dtype)
    k, v = (randn(g, (keys, kv, dim), dtype) for _ in range(2))
    return q, k, v, *(torch.tensor([0, n], dtype=torch.int32, device=DEV) for n in (queries, keys))


@pytest.mark.parametrize("silent", [1, 2, 3, 6, 9, 14, -1])
@pytest.mark.parametrize("queries,keys,heads,kv,dim,dtype", [(1000, 1000, 8, 2, 128, torch.bfloat16),
                                                             (900, 1300, 3, 3, 64, torch.float16),
                                                             (20, 9000, 8, 2, 64, torch.bfloat16),
                                                             (300, 9001, 2, 1, 96, torch.float16)])
def test_waits_run_out(opa, monkeypatch, queries, keys, heads, kv, dim, dtype, silent):
    """Copies that end before a block's N-th tile; for -1 a warp that does not come where parts are
    joined, which only calls that cut keys do."""
    args = inputs(queries, keys, heads, kv, dim, dtype)
    with opa.Context(0) as ctx:
        want = ctx.attention(*args)[1]
        ctx.check()
    monkeypatch.setenv("OPATTR_FAULT", f"prompt:{silent}")
    with opa.Context(0) as ctx:
        first = ctx.attention(*args)[1]
        monkeypatch.delenv("OPATTR_FAULT")
        if silent < 0 and queries > 500:
            ctx.check()
            assert torch.equal(first, want)
        else:
            ctx.attention(*args)                         # begins nothing: what is left behind is not used
            with pytest.raises(opa.OpattrError) as e:
                ctx.check()
            assert e.value.status == opa.E_TIMEOUT
        for _ in range(2):
            assert torch.equal(ctx.attention(*args)[1], want)
            ctx.check()


def test_wait_for_a_long_item(opa):
    """One query over 800 million keys, of which the first and the last thousand matter, among two
    thousand sequences that have none: one item of one block, whose waits last longer than
    those of any ordinary call."""
    n, seqs = 800_000_000, 2100
    kv = torch.zeros((n, 1, 8), dtype=torch.bfloat16, device=DEV)
    kv[:, 0, 0] = -200.0
    kv[:1000, 0, 0], kv[-1000:, 0, 0] = 0.0, 0.0
    kv[:1000, 0, 1], kv[-1000:, 0, 1] = 1.0, 3.0
    q = torch.zeros((1, 1, 8), dtype=torch.bfloat16, device=DEV)
    q[:, :, 0] = 1.0
    ends = [torch.tensor([0] + [x] * seqs, dtype=torch.int32, device=DEV) for x in (1, n)]
    with opa.Context(0) as ctx:
        _, out, lse = ctx.attention(q, kv, kv, *ends, causal=False, scale=1.0, need_lse=True)
        ctx.check()
    assert out.flatten().tolist() == [0.0, 2.0] + [0.0] * 6
    assert abs(float(lse) - 7.600902459542082) < 1e-5          # log of 2,000

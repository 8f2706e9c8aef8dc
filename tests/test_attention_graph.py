"""The attention operators and the cache's calls in captured graphs (GPU)."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
import tracegen  # noqa: E402
from attn_util import randn  # noqa: E402

DEV = "cuda:0"
BF = torch.bfloat16


@pytest.fixture(scope="module")
def opa():
    import paper_2609_11938_gb300 as opa
    return opa


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def i32(*x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def test_graph_outlives_its_scratch(opa):
    """A token step and a prompt over many keys, captured; larger calls and a join on the
    same context; then the replay, beside tensors in whatever memory was let go."""
    g = gen(41)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s), opa.Context(0, stream=s) as ctx:
        c = ctx.cache(700, 16, 2, 64, 3, 600)
        lens = [9000, 40, 333]
        k, v = (randn(g, (sum(lens), 2, 64), BF) for _ in range(2))
        seqs, back = i32(0, 1, 2), i32(*lens)
        ctx.cache_append(c, seqs, i32(0, 9000, 9040, 9373), k, v)
        k1, v1 = (randn(g, (3, 2, 64), BF) for _ in range(2))
        q1, off1 = randn(g, (3, 8, 64), BF), i32(0, 1, 2, 3)
        q, off, koff = randn(g, (20, 8, 64), BF), i32(0, 20), i32(0, 9373)

        def step():
            ctx.cache_append(c, seqs, off1, k1, v1)
            _, out, _ = ctx.cache_attention(c, seqs, q1)
            ctx.cache_trim(c, seqs, back)
            return out, ctx.attention(q, k, v, off, koff)[1]

        want = [x.clone() for x in step()]
        ctx.check()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            got = step()
        # larger calls, each past the scratch of those before it
        wide = [randn(g, (n, h, 128), BF) for n, h in ((20, 8), (9000, 1), (9000, 1))]
        ctx.attention(*wide, off, i32(0, 9000))
        ctx.cache_compact(ctx.cache(6_000_000, 16, 1, 8, 1, 1))
        ctx.check()
        ctx.join(opa.to_device(tracegen.generate("tiny")))
        others = [torch.full((n << 18,), 7.0, device=DEV) for n in [40, 20, 10, 4, 1] * 4]
        for x in got:
            x.zero_()
        for _ in range(2):
            graph.replay()
            ctx.check()
            assert all(torch.equal(a, b) for a, b in zip(got, want))
        assert c.length.tolist() == lens
        assert all(bool((x == 7).all()) for x in others)
        assert all(torch.equal(a, b) for a, b in zip(step(), want))
        ctx.check()
        del graph


@pytest.mark.parametrize("first", [True, False])
def test_no_scratch_under_capture(opa, first):
    """A captured call that has no scratch yet, the context's first or one larger than those
    before it, is refused; the capture and the context go on."""
    g = gen(42)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s), opa.Context(0, stream=s) as ctx:
        q = randn(g, (20, 8, 64), BF)
        k, v = (randn(g, (9000, 2, 64), BF) for _ in range(2))
        off, koff = i32(0, 20), i32(0, 9000)
        if not first:
            ctx.attention(q, q, q, off)
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            with pytest.raises(opa.OpattrError) as e:
                ctx.attention(q, k, v, off, koff)
            other = q + 1
        assert e.value.status == opa.E_OOM
        other.zero_()
        graph.replay()
        assert torch.equal(other, q + 1)
        a = ctx.attention(q, k, v, off, koff)[1]
        ctx.check()
        with torch.cuda.graph(torch.cuda.CUDAGraph(), stream=s):
            ctx.attention(q, k, v, off, koff)
        assert torch.equal(ctx.attention(q, k, v, off, koff)[1], a)
        ctx.check()


def test_timing_and_capture(opa):
    """With timing on, captured launches are not timed, those before and after it are."""
    g = gen(43)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s), opa.Context(0, stream=s) as ctx:
        q, k, v = (randn(g, (200, 2, 64), BF) for _ in range(3))
        off = i32(0, 200)
        ctx.set_timing(True)
        want = ctx.attention(q, k, v, off)[1]
        ctx.check()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            got = ctx.attention(q, k, v, off)[1]
        ctx.check()
        graph.replay()
        again = ctx.attention(q, k, v, off)[1]
        ctx.check()
        assert torch.equal(got, want) and torch.equal(again, want)
        ms, launches = ctx.timing_report()["prompt"]
        assert launches == 2 and 0 < ms < 1e3


@pytest.mark.parametrize("queries,keys", [(200, 200), (1, 1), (20, 300), (30, 0), (2, 9000)])
def test_one_sequence_without_offsets(opa, queries, keys):
    """A call without offsets does not wait for the device either, and can be captured."""
    g = gen(44)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s), opa.Context(0, stream=s) as ctx:
        q, k, v = (randn(g, (n, 2, 64), BF) for n in (queries, keys, keys))
        off = [i32(0, queries), i32(0, keys)]
        want = ctx.attention(q, k, v, *off)[1]
        ctx.check()
        torch.cuda.set_sync_debug_mode("error")
        try:
            got = ctx.attention(q, k, v)[1]
        finally:
            torch.cuda.set_sync_debug_mode("default")
        ctx.check()
        assert torch.equal(got, want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            got = ctx.attention(q, k, v)[1]
        got.fill_(7)
        graph.replay()
        ctx.check()
        assert torch.equal(got, want)

"""The paged cache in 8 bits (GPU): its state and pools, whole, against a model of its
definition, call after call; attention over it against 64 bits."""
import math
import random

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from attn_util import assert_within, randn  # noqa: E402
from window_util import Model8, attend8, near_mask, stands_for  # noqa: E402

DEV = "cuda:0"
BF, HF, E4 = torch.bfloat16, torch.float16, torch.float8_e4m3fn


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


def fresh(ctx, n_pages, page, heads, dim, n_seqs, per):
    """An empty cache whose pools hold something that shows where nobody writes."""
    c = ctx.cache(n_pages, page, heads, dim, n_seqs, per, E4)
    c.k_pages.view(torch.uint8).fill_(0x55)
    c.v_pages.view(torch.uint8).fill_(0xd3)
    c.k_scales.fill_(3.0)
    c.v_scales.fill_(math.nan)
    return c, Model8(c)


def host(x):
    return x.double().cpu().numpy()


def both(ctx, c, m, seqs, counts, k, v):
    ctx.cache_append(c, i32(seqs), offsets(counts), k, v)
    m.append(seqs, counts, host(k), host(v))


def check_attention(ctx, c, q, seqs, window=None, sinks=0, scale=None):
    _, out, lse = ctx.cache_attention(c, i32(seqs), q, need_lse=True, window=window, sinks=sinks, scale=scale)
    ctx.check()
    for i, s in enumerate(seqs):
        k, v = stands_for(c, s)
        n = k.shape[0]
        seen = near_mask(1, n, window or n, sinks, DEV) if n else torch.ones((1, 0), dtype=torch.bool, device=DEV)
        want, wl, lim, ll = attend8(q[i:i + 1], k, v, q.shape[2] ** -0.5 if scale is None else scale, seen)
        assert_within(out[i:i + 1], want, lim, f"out of sequence {s} ({n} tokens)")
        assert_within(lse[i:i + 1], wl, ll, f"lse of sequence {s} ({n} tokens)")
    return out, lse


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("seed,page,heads,dim", [(0, 16, 1, 16), (1, 16, 3, 64), (2, 32, 2, 48), (3, 128, 1, 128), (4, 64, 2, 112)])
def test_calls_in_any_order(ctx, dtype, seed, page, heads, dim):
    rng, g = random.Random(seed), gen(seed)
    n_seqs, per, n_pages = 9, 6, 40
    c, m = fresh(ctx, n_pages, page, heads, dim, n_seqs, per)
    for turn in range(60):
        what = rng.choice(["append", "append", "append", "fork", "trim", "trim", "compact"])
        if what == "append":
            seqs = rng.sample(range(n_seqs), rng.randint(1, n_seqs))
            counts = [min(rng.choice([0, 1, 1, 5, 16, page, 2 * page + 1]), per * page - m.length[s]) for s in seqs]
            if sum(-(-(m.length[s] + n) // page) + 1 for s, n in zip(seqs, counts)) > m.refs.count(0):
                continue
            spread = 2.0 ** rng.randint(-6, 6)
            k, v = (randn(g, (sum(counts), heads, dim), dtype, spread) for _ in range(2))
            both(ctx, c, m, seqs, counts, k, v)
        elif what == "fork":
            empty = [s for s in range(n_seqs) if m.length[s] == 0]
            full = [s for s in range(n_seqs) if m.length[s] > 0]
            if not empty or not full:
                continue
            dst = rng.sample(empty, rng.randint(1, len(empty)))
            src = [rng.choice(full) for _ in dst]
            ctx.cache_fork(c, i32(src), i32(dst))
            m.fork(src, dst)
        elif what == "trim":
            seqs = rng.sample(range(n_seqs), rng.randint(1, 4))
            to = [rng.choice([0, m.length[s] // 2, max(0, m.length[s] - 1), m.length[s]]) for s in seqs]
            ctx.cache_trim(c, i32(seqs), i32(to))
            m.trim(seqs, to)
        else:
            _, live = ctx.cache_compact(c)
            assert int(live) == m.compact()
        ctx.check()
        m.same(c)
        if turn % 10 == 9:
            check_attention(ctx, c, randn(g, (n_seqs, 2 * heads, dim), dtype, 1.5), list(range(n_seqs)))


@pytest.mark.parametrize("dtype", [BF, HF])
def test_rounding(ctx, dtype):
    """Blocks of every size of numbers: zeros, the least and the largest, powers of two and
    their neighbours, ties, and what is not finite."""
    c, m = fresh(ctx, 40, 16, 2, 32, 40, 1)
    top = torch.finfo(dtype).max
    tiny = torch.finfo(dtype).smallest_normal
    rows = []
    for x in (0.0, -0.0, tiny, tiny / 8, top, -top, 448.0, 449.0, 1.75, 1.7578125, 2.0 ** -9, 240.0, 464.0, math.inf, -math.inf, math.nan, 1e-30):
        r = torch.zeros((16, 2, 32), dtype=torch.float64, device=DEV)
        r[0, 0, 0] = x
        r[1, 0, :] = x / 3 if math.isfinite(x) else 1.0
        r[2, 1, 5] = x
        r[3, 1, :] = torch.linspace(-1, 1, 32, device=DEV)
        # ties between neighbouring codes of a block whose scale is 1
        r[4, 0, :16] = torch.arange(16, device=DEV) * 0.0625 + 1.0
        r[5, 0, :16] = torch.arange(16, device=DEV) * 2.0 ** -10
        rows.append(r.to(dtype))
    n = len(rows)
    k = torch.cat(rows)
    both(ctx, c, m, list(range(n)), [16] * n, k, -k)
    # the same one token at a time
    for t in range(16):
        step = torch.cat([r[t:t + 1] for r in rows])
        both(ctx, c, m, list(range(n, 2 * n)), [1] * n, step, -step)
    ctx.check()
    m.same(c)


def test_scales_grow(ctx):
    """Token by token, each far above or below those before; codes that fall below the least one."""
    c, m = fresh(ctx, 9, 32, 1, 16, 3, 3)
    g = gen(2)
    for t in range(70):
        k, v = (randn(g, (3, 1, 16), BF, 2.0 ** ((7 * t) % 23 - 8)) for _ in range(2))
        both(ctx, c, m, [0, 1, 2], [1, 1, 1], k, v)
    ctx.check()
    m.same(c)


def test_scales_of_others(ctx):
    """A scale that is no power of two is taken as it is."""
    c, m = fresh(ctx, 4, 16, 1, 32, 2, 2)
    g = gen(4)
    k = randn(g, (10, 1, 32), BF)
    both(ctx, c, m, [0, 1], [5, 5], k, k)
    for scales, own in zip((c.k_scales, c.v_scales), m.scales):
        for at, x in ((0, 0.0371), (1, 1e-5)):
            scales[at], own[at] = x, float(torch.tensor(x, dtype=torch.float32))
    k = randn(g, (6, 1, 32), BF)
    both(ctx, c, m, [0, 1], [3, 3], k, k)
    ctx.check()
    m.same(c)
    check_attention(ctx, c, randn(g, (2, 4, 32), HF), [0, 1])


@pytest.mark.parametrize("page,heads,dim", [(32, 2, 64), (64, 1, 128)])
def test_shared_page_that_was_shortened(ctx, page, heads, dim):
    """Sequences that hold one page begin to write at different places of it, in one call."""
    g = gen(page)
    c, m = fresh(ctx, 30, page, heads, dim, 8, 3)
    k, v = (randn(g, (page - 3, heads, dim), BF) for _ in range(2))
    both(ctx, c, m, [0], [page - 3], k, v)
    ctx.cache_fork(c, i32([0] * 5), i32([1, 2, 3, 4, 5]))
    m.fork([0] * 5, [1, 2, 3, 4, 5])
    to = [page - 3, page - 5, 17, 16, 5, 3]
    for order in ([0, 1, 2, 3, 4, 5], [5, 2, 4, 0, 3, 1]):
        ctx.cache_trim(c, i32(order), i32([to[s] for s in order]))
        m.trim(order, [to[s] for s in order])
        counts = [7, 1, 20, 3, 1, 40]
        k, v = (randn(g, (sum(counts), heads, dim), BF, 5.0) for _ in range(2))
        both(ctx, c, m, order, counts, k, v)
        ctx.check()
        m.same(c)
        for s in range(6):
            if m.length[s]:
                ctx.cache_trim(c, i32([s]))
                m.trim([s], [0])
        k, v = (randn(g, (page - 3, heads, dim), BF) for _ in range(2))
        both(ctx, c, m, [0], [page - 3], k, v)
        ctx.cache_fork(c, i32([0] * 5), i32([1, 2, 3, 4, 5]))
        m.fork([0] * 5, [1, 2, 3, 4, 5])


def test_many_sequences(ctx):
    """More sequences than a warp looks up at a time, empty ones among them."""
    g, rng = gen(6), random.Random(6)
    n = 150
    c, m = fresh(ctx, 900, 16, 1, 32, n, 6)
    for _ in range(2):
        counts = [rng.choice([0, 1, 2, 15, 16, 17, 40]) for _ in range(n)]
        seqs = rng.sample(range(n), n)
        k, v = (randn(g, (sum(counts), 1, 32), HF) for _ in range(2))
        both(ctx, c, m, seqs, counts, k, v)
    ctx.check()
    m.same(c)


def test_refused_calls_change_nothing(ctx):
    import paper_2609_11938_gb300 as opa
    g = gen(1)
    c, m = fresh(ctx, 4, 16, 1, 32, 3, 4)
    k = randn(g, (20, 1, 32), BF)
    both(ctx, c, m, [0], [20], k, k)
    ctx.check()
    for seqs, counts, status in (([1, 1], [1, 1], opa.E_INVALID_ARG), ([3], [1], opa.E_INVALID_ARG), ([0], [60], opa.E_INVALID_ARG),
                                 ([1, 2], [30, 30], opa.E_PAGES)):
        k = randn(g, (sum(counts), 1, 32), BF)
        ctx.cache_append(c, i32(seqs), offsets(counts), k, k)
        with pytest.raises(opa.OpattrError) as e:
            ctx.check()
        assert e.value.status == status
        m.same(c)


# ---------------------------------------------------------------- attention
LENS = [1, 0, 15, 16, 17, 127, 128, 129, 255, 700, 1025, 2600]


def filled(ctx, lens, page, kv, dim, dtype, seed):
    g = gen(seed)
    per = max(1, -(-max(lens) // page))
    c = ctx.cache(sum(-(-n // page) for n in lens) + 3, page, kv, dim, len(lens), per, E4)
    # what lies past a sequence's end is NaN, and so are the scales of blocks that nobody wrote
    c.k_pages.view(torch.uint8).fill_(0x7f)
    c.v_pages.view(torch.uint8).fill_(0xff)
    c.k_scales.fill_(math.nan)
    c.v_scales.fill_(math.inf)
    k, v = (randn(g, (sum(lens), kv, dim), dtype) + randn(g, (1, kv, dim), dtype) for _ in range(2))
    ctx.cache_append(c, i32(range(len(lens))), offsets(lens), k, v)
    return c, g


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dim,heads,kv,page", [(64, 12, 12, 16), (128, 8, 2, 32), (128, 24, 2, 64), (64, 11, 1, 16), (16, 3, 3, 128), (48, 4, 2, 16),
                                               (80, 20, 4, 32), (112, 17, 1, 1024)])
@pytest.mark.parametrize("window,sinks", [(None, 0), (1, 0), (16, 1), (100, 4), (1000, 200), (2 ** 31 - 1, 3)])
def test_attention(ctx, dtype, dim, heads, kv, page, window, sinks):
    c, g = filled(ctx, LENS, page, kv, dim, dtype, dim + heads)
    seqs = list(range(len(LENS))) + [9, 11, 11]
    check_attention(ctx, c, randn(g, (len(seqs), heads, dim), dtype, 1.5), seqs, window, sinks)


@pytest.mark.parametrize("dim,heads,dtype", [(64, 4, BF), (48, 48, HF), (128, 8, HF), (96, 40, BF)])
@pytest.mark.parametrize("window,sinks", [(None, 0), (100, 20), (3000, 1)])
def test_many_pairs(ctx, dim, heads, dtype, window, sinks):
    """So many sequences and key heads that each warp has its own, with some among them that many warps share."""
    rng = random.Random(dim)
    lens = [rng.choice([0, 1, 15, 33, rng.randint(1, 300)]) for _ in range(490)] + [9000, 3001, 700]
    rng.shuffle(lens)
    c, g = filled(ctx, lens, 32, 4, dim, dtype, dim)
    seqs = list(range(len(lens)))
    q = randn(g, (len(lens), heads, dim), dtype, 1.5)
    _, out, lse = ctx.cache_attention(c, None, q, need_lse=True, window=window, sinks=sinks)
    again = ctx.cache_attention(c, i32(seqs), q, need_lse=True, window=window, sinks=sinks)
    ctx.check()
    assert torch.equal(out, again[1]) and torch.equal(lse, again[2])
    for s in [i for i, n in enumerate(lens) if n > 600] + rng.sample(seqs, 40):
        k, v = stands_for(c, s)
        n = k.shape[0]
        seen = near_mask(1, n, window or n, sinks, DEV) if n else torch.ones((1, 0), dtype=torch.bool, device=DEV)
        want, wl, lim, ll = attend8(q[s:s + 1], k, v, dim ** -0.5, seen)
        assert_within(out[s:s + 1], want, lim, f"out of sequence {s} ({n} tokens)")
        assert_within(lse[s:s + 1], wl, ll, f"lse of sequence {s} ({n} tokens)")


@pytest.mark.parametrize("dtype", [BF, HF])
def test_scales_far_apart(ctx, dtype):
    """Blocks whose scales are many powers of two apart, and queries of every size."""
    g = gen(8)
    lens = [400, 33]
    c = ctx.cache(40, 16, 2, 64, 2, 30, E4)
    grow = torch.exp2(torch.arange(sum(lens), device=DEV).float().div(16).floor() % 25 - 12)[:, None, None]
    limit = 1.0 if dtype is BF else 0.05
    k, v = ((randn(g, (sum(lens), 2, 64), torch.float32) * grow * s).to(dtype) for s in (2.0 ** -9, limit))
    ctx.cache_append(c, i32([0, 1]), offsets(lens), k, v)
    q = randn(g, (2, 6, 64), torch.float32)
    q[0] *= torch.exp2(-torch.arange(64, device=DEV).float() / 3)
    for spread in (2.0 ** -10, 1.0, 2.0 ** 5):
        check_attention(ctx, c, (q * spread).to(dtype), [0, 1])
        check_attention(ctx, c, (q * spread).to(dtype), [0, 1], window=100, sinks=20)


def test_queries_at_the_ends_of_the_range(ctx):
    """bfloat16 queries near its largest and its least values, and rows of zeros."""
    c, g = filled(ctx, [200, 90, 31], 16, 1, 32, BF, 5)
    q = randn(g, (3, 4, 32), torch.float32)
    q[0] *= 2.0 ** 120
    q[1] *= 2.0 ** -130
    q[2] = 0
    check_attention(ctx, c, q[:1].to(BF), [0], scale=2.0 ** -122)
    check_attention(ctx, c, q.to(BF)[1:], [1, 2])


@pytest.mark.parametrize("dtype", [BF, HF])
def test_not_finite(ctx, dtype):
    """A key or value that is seen makes its rows NaN, one that is not seen does nothing."""
    g = gen(12)
    n, at = 300, 37
    c = ctx.cache(20, 16, 2, 32, 1, 20, E4)
    k, v = (randn(g, (n, 2, 32), dtype) for _ in range(2))
    k[at, 0, 3], v[at + 1, 1, 5] = math.inf, math.nan
    ctx.cache_append(c, i32([0]), i32([0, n]), k, v)
    q = randn(g, (1, 4, 32), dtype)
    out, lse = ctx.cache_attention(c, None, q, need_lse=True)[1:]
    assert out[0, :2].isnan().all() and lse[0, :2].isnan().all()
    assert lse[0, 2:].isfinite().all() and out[0, 2:, 5].isnan().all() and out[0, 2:].isnan().sum() == 2
    check_attention(ctx, c, q, [0], window=n - at - 2)
    check_attention(ctx, c, q, [0], window=100, sinks=at)


def test_parts_are_joined_in_order(ctx):
    c, g = filled(ctx, [60_000, 20_000], 64, 1, 128, BF, 21)
    q = randn(g, (2, 8, 128), BF, 1.5)
    a = check_attention(ctx, c, q, [0, 1])
    for _ in range(3):
        b = ctx.cache_attention(c, i32([0, 1]), q, need_lse=True)
        assert torch.equal(a[0], b[1]) and torch.equal(a[1], b[2])


def test_pools_past_32_bits(ctx):
    """Pages whose first byte lies past 2^32."""
    page, kv, dim = 1024, 8, 128
    n_pages = (1 << 32) // (page * kv * dim) + 2
    c = ctx.cache(n_pages, page, kv, dim, 1, 2, E4)
    c.refs.fill_(1)
    c.refs[-2:] = 0
    g = gen(1)
    n = 1500
    k, v = (randn(g, (n, kv, dim), BF) for _ in range(2))
    ctx.cache_append(c, i32([0]), i32([0, n]), k, v)
    ctx.check()
    assert c.table.tolist() == [[n_pages - 2, n_pages - 1]]
    got = stands_for(c, 0)
    for x, y in zip(got, (k, v)):
        assert ((x - y.double()).abs() <= y.double().abs() * 2.0 ** -4 * 1.001 + 2.0 ** -9 * 0.02).all()
    assert not c.k_pages.view(torch.uint8)[:-2].any() and not c.k_scales[:-2].any()
    check_attention(ctx, c, randn(g, (1, 16, 128), BF), [0])
    check_attention(ctx, c, randn(g, (1, 16, 128), HF), [0], window=600, sinks=4)


def test_rows_of_any_stride(ctx):
    g = gen(7)
    c, m = fresh(ctx, 12, 16, 2, 48, 2, 5)
    big = randn(g, (70, 5, 3 * 48), HF)
    k, v = big[:, 1:3, :48], big[:, 3:4, 96:].expand(70, 2, 48)
    both(ctx, c, m, [1, 0], [30, 40], k, v)
    ctx.check()
    m.same(c)
    q = big[:2, 1:5, 48:96]
    out = torch.full((2, 6, 48), 7.0, dtype=HF, device=DEV)
    _, got, _ = ctx.cache_attention(c, i32([1, 0]), q, out=out[:, 1:5])
    ctx.check()
    want = ctx.cache_attention(c, i32([1, 0]), q.contiguous())[1]
    assert torch.equal(got, want) and (out[:, 0] == 7).all() and (out[:, 5] == 7).all()


def test_captured_steps(ctx):
    """A serving step over each kind of cache, captured and replayed, beside eager calls."""
    import paper_2609_11938_gb300 as opa
    g = gen(30)
    lens = [40, 129, 15]
    n, kv, dim = len(lens), 2, 64
    for dtype, e4 in ((BF, True), (HF, True), (BF, False)):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream), opa.Context(0, stream=stream) as own:
            caches = [own.cache(40, 16, kv, dim, n, 12, E4 if e4 else dtype) for _ in range(2)]
            k, v = (randn(g, (sum(lens), kv, dim), dtype) for _ in range(2))
            q, k1, v1 = (torch.empty((n, h, dim), dtype=dtype, device=DEV) for h in (4, kv, kv))
            prompt, seqs, one = offsets(lens), i32(range(n)), offsets([1] * n)
            qp = randn(g, (sum(lens), 4, dim), dtype)

            def step(c):
                own.cache_append(c, seqs, one, k1, v1)
                a = own.attention(qp, k, v, prompt, window=21, sinks=2)[1]
                return own.cache_attention(c, seqs, q, window=50, sinks=3, need_lse=True)[1:] + (a,)

            for c in caches:
                own.cache_append(c, seqs, prompt, k, v)
            for x in (q, k1, v1):
                x.copy_(randn(g, x.shape, dtype))
            step(caches[0])
            step(caches[1])
            own.check()
            stream.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                got = step(caches[0])
            for _ in range(5):
                for x in (q, k1, v1):
                    x.copy_(randn(g, x.shape, dtype))
                graph.replay()
                want = step(caches[1])
                own.check()
                assert all(torch.equal(a, b) for a, b in zip(got, want))
                assert torch.equal(caches[0].length, caches[1].length)
                assert torch.equal(caches[0].k_pages.view(torch.uint8), caches[1].k_pages.view(torch.uint8))
            stream.synchronize()


def test_served_together(ctx):
    """Prompts through a window, their keys and values into 8 bits, tokens on top of them,
    forked, shortened, compacted: every step's results from what the cache holds."""
    g = gen(40)
    lens, kv, dim, heads = [200, 31, 90], 2, 64, 8
    c, m = fresh(ctx, 60, 16, kv, dim, 6, 20)
    q = randn(g, (sum(lens), heads, dim), BF, 1.5)
    k, v = (randn(g, (sum(lens), kv, dim), BF) for _ in range(2))
    ctx.attention(q, k, v, offsets(lens), window=64, sinks=4)
    both(ctx, c, m, [0, 1, 2], lens, k, v)
    live = [0, 1, 2]
    for t in range(12):
        k, v = (randn(g, (len(live), kv, dim), BF, 1.0 + t / 3) for _ in range(2))
        both(ctx, c, m, live, [1] * len(live), k, v)
        check_attention(ctx, c, randn(g, (len(live), heads, dim), BF, 1.5), live, 64, 4)
        if t == 4:
            ctx.cache_fork(c, i32([0, 0]), i32([3, 4]))
            m.fork([0, 0], [3, 4])
            live = [0, 1, 2, 3, 4]
        if t == 8:
            ctx.cache_trim(c, i32([1, 3]))
            m.trim([1, 3], [0, 0])
            live = [0, 2, 4]
            assert int(ctx.cache_compact(c)[1]) == m.compact()
        ctx.check()
        m.same(c)

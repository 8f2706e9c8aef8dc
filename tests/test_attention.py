"""Attention over packed prompts and over the paged cache (GPU), against its
definition in 64 bits: types, head layouts, lengths about the tiles' sizes, rows
that see nothing, strides, values outside a row's mask that are not finite."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from attn_util import assert_within, attend, causal_mask, randn  # noqa: E402

DEV = "cuda:0"
BF, HF = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def opa():
    import paper_2609_11938_gb300 as opa
    return opa


@pytest.fixture(scope="module")
def ctx(opa):
    with opa.Context(0) as c:
        yield c


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def offsets(lens):
    return torch.tensor([0] + list(torch.tensor(lens).cumsum(0)) if lens else [0], dtype=torch.int32, device=DEV)


def check_prompt(ctx, q, k, v, lq, lk, causal, scale=None, **kw):
    scale_ = q.shape[2] ** -0.5 if scale is None else scale
    _, out, lse = ctx.attention(q, k, v, offsets(lq), None if lk is None else offsets(lk), causal=causal, scale=scale,
                                need_lse=True, **kw)
    ctx.check()
    a = b = 0
    for i, n in enumerate(lq):
        m = n if lk is None else lk[i]
        seen = causal_mask(n, m, DEV) if causal else torch.ones((n, m), dtype=torch.bool, device=DEV)
        want, wl, lim, ll = attend(q[a:a + n], k[b:b + m], v[b:b + m], scale_, seen)
        assert_within(out[a:a + n], want, lim, f"out of sequence {i} ({n} queries, {m} keys)")
        assert_within(lse[a:a + n], wl, ll, f"lse of sequence {i} ({n} queries, {m} keys)")
        a, b = a + n, b + m
    return out, lse


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dim", [8, 64, 72, 128])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lens", [[1], [2, 1, 3], [127, 128, 129], [255, 0, 257], [640, 1, 63]])
def test_prompt_lengths(ctx, dtype, dim, causal, lens):
    g = gen(sum(lens) * 131 + dim)
    n = sum(lens)
    q, k, v = (randn(g, (n, h, dim), dtype) for h in (4, 2, 2))
    check_prompt(ctx, q, k, v, lens, None, causal)


@pytest.mark.parametrize("heads,kv", [(1, 1), (3, 3), (7, 1), (12, 4), (16, 16), (40, 8), (13, 1), (26, 2), (48, 1),
                                      (120, 1), (131, 1), (256, 2)])
def test_prompt_heads(ctx, heads, kv):
    g = gen(heads)
    lens = [150, 33]
    q, k, v = (randn(g, (183, h, 64), BF) for h in (heads, kv, kv))
    check_prompt(ctx, q, k, v, lens, None, True)


@pytest.mark.parametrize("dtype,dim", [(BF, 128), (HF, 64), (BF, 40)])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lq,lk", [([5], [300]), ([300], [5]), ([1, 130, 40], [1000, 131, 0]), ([0, 200], [7, 200]),
                                   ([256, 129], [511, 385])])
def test_prompt_pieces(ctx, dtype, dim, causal, lq, lk):
    """Keys begin before the queries, or after the first of them (rows that see
    nothing), or there are none."""
    g = gen(sum(lq) + 3 * sum(lk) + dim)
    q = randn(g, (sum(lq), 6, dim), dtype)
    k, v = (randn(g, (sum(lk), 3, dim), dtype) for _ in range(2))
    out, lse = check_prompt(ctx, q, k, v, lq, lk, causal)
    if causal and lq == [300]:
        assert (out[:295] == 0).all() and (lse[:295] == -math.inf).all()


@pytest.mark.parametrize("heads,kv", [(2, 2), (6, 2), (4, 1)])
def test_prompt_neighbours(ctx, heads, kv):
    """A sequence's bits do not depend on the queries, keys and values packed beside it."""
    g = gen(21)
    lens = [137, 300, 41]
    q, k, v = (randn(g, (478, h, 64), BF) for h in (heads, kv, kv))
    want = ctx.attention(q, k, v, offsets(lens))[1][137:437]
    for x in (q, k, v):
        x[:137], x[437:] = 50.0, -80.0
    assert torch.equal(ctx.attention(q, k, v, offsets(lens))[1][137:437], want)


def test_prompt_long(ctx):
    g = gen(5)
    n = 5001
    q, k, v = (randn(g, (n, h, 128), BF) for h in (2, 1, 1))
    check_prompt(ctx, q, k, v, [n], None, True)


@pytest.mark.parametrize("dtype,dim,heads,kv", [(BF, 128, 4, 2), (HF, 64, 3, 1), (BF, 96, 5, 5)])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lq,lk", [([1], [20_000]), ([300, 1, 40], [9001, 30, 5000]), ([0, 257], [3, 4999]), ([200], [4100])])
def test_prompt_few_queries_many_keys(ctx, dtype, dim, heads, kv, causal, lq, lk):
    """Keys cut into pieces, their parts joined; twice, for the counts left behind."""
    g = gen(sum(lk) + dim)
    q = randn(g, (sum(lq), heads, dim), dtype)
    k, v = (randn(g, (sum(lk), kv, dim), dtype) for _ in range(2))
    first, _ = check_prompt(ctx, q, k, v, lq, lk, causal)
    assert torch.equal(check_prompt(ctx, q, k, v, lq, lk, causal)[0], first)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype,dim,heads,kv,seqs,queries,keys", [(BF, 64, 8, 1, 40, 30, 6000), (HF, 128, 6, 3, 3, 400, 9000),
                                                                  (BF, 80, 7, 1, 70, 3, 9000), (BF, 128, 2, 2, 1, 900, 7000)])
def test_prompt_equal_runs(ctx, causal, dtype, dim, heads, kv, seqs, queries, keys):
    """Runs of keys that hold several items and parts of some, beside sequences without
    queries or keys; then with a value that one query sees alone and that is not finite."""
    g = gen(seqs * 7 + dim)
    rnd = torch.Generator().manual_seed(seqs)
    lq = [int(x) for x in torch.randint(0 if seqs > 1 else queries, queries + 1, (seqs,), generator=rnd)]
    lk = [int(x) for x in torch.randint(keys // 2 if seqs < 5 else 0, keys + 1, (seqs,), generator=rnd)]
    if seqs > 5:
        lk[3], lq[5] = 0, 0
    q = randn(g, (sum(lq), heads, dim), dtype)
    k, v = (randn(g, (sum(lk), kv, dim), dtype) for _ in range(2))
    first, _ = check_prompt(ctx, q, k, v, lq, lk, causal)
    assert torch.equal(check_prompt(ctx, q, k, v, lq, lk, causal)[0], first)
    n, m = lq[-1], lk[-1]
    if causal and n > 1 and m > 1:
        want, _, lim, _ = attend(q[-n:], k[-m:], v[-m:], dim ** -0.5, causal_mask(n, m, DEV))
        v[-1] = math.inf
        out = ctx.attention(q, k, v, offsets(lq), offsets(lk))[1]
        ctx.check()
        assert torch.equal(out[:-n], first[:-n])
        assert_within(out[-n:-1], want[:-1], lim[:-1], "rows that do not see it")
        assert not torch.isfinite(out[-1]).any()


def test_prompt_rising_scores(ctx):
    """Scores that rise along the keys: the running maximum moves at every tile,
    by more and by less than what the accumulator is rescaled for."""
    g = gen(6)
    for step in (0.01, 0.05, 0.5):
        n = 700
        q = torch.ones((n, 2, 64), dtype=BF, device=DEV)
        k = (torch.arange(n, device=DEV) * step)[:, None, None].expand(n, 2, 64).to(BF).contiguous()
        v = randn(g, (n, 2, 64), BF)
        check_prompt(ctx, q, k, v, [n], None, True, scale=1 / 64)
        check_prompt(ctx, q, k.flip(0).contiguous(), v, [n], None, False, scale=1 / 64)


@pytest.mark.parametrize("scale", [0.0, -0.3, 2.0])
def test_prompt_scale(ctx, scale):
    g = gen(7)
    q, k, v = (randn(g, (200, 2, 64), HF) for _ in range(3))
    check_prompt(ctx, q, k, v, [200], None, True, scale=scale)


def test_prompt_views(ctx):
    """Queries, keys and values as views of one projection, heads before tokens,
    and rows with room between them; an output that is a view as well."""
    g = gen(8)
    n, H, G, D = 190, 4, 2, 64
    qkv = randn(g, (n, (H + 2 * G) * D), BF)
    q, k, v = (x.view(n, -1, D) for x in qkv.split([H * D, G * D, G * D], 1))
    room = torch.full((n, H, 2 * D), 7.0, dtype=BF, device=DEV)
    out, _ = check_prompt(ctx, q, k, v, [100, 90], None, True, out=room[:, :, :D])
    assert out.data_ptr() == room.data_ptr() and (room[:, :, D:] == 7).all()
    hq, hk, hv = (randn(g, (h, n, D), BF).transpose(0, 1) for h in (H, G, G))
    check_prompt(ctx, hq, hk, hv, [n], None, True)
    one = randn(g, (n, 1, D), BF)
    check_prompt(ctx, q, one.expand(n, G, D), v, [n], None, False)        # one key head for all
    check_prompt(ctx, one.expand(n, H, D), k, v, [n], None, True)         # one query for all heads


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_prompt_masked_values(ctx, dtype, bad):
    """Keys and values past a row's mask that are not finite: in the sequence
    after it, and later in its own."""
    g = gen(9)
    lens = [100, 150, 20]
    q, k, v = (randn(g, (270, 2, 64), dtype) for _ in range(3))
    k2, v2 = k.clone(), v.clone()
    k2[100:], v2[100:] = bad, bad                      # every row of the others
    _, out, lse = ctx.attention(q, k2, v2, offsets(lens))
    _, want, _ = ctx.attention(q, k, v, offsets(lens))
    ctx.check()
    assert torch.equal(out[:100], want[:100])
    k2, v2 = k.clone(), v.clone()
    k2[190, 0], v2[190, 0] = bad, bad                  # token 90 of the second, one head of two
    _, out, _ = ctx.attention(q, k2, v2, offsets(lens))
    ctx.check()
    for a, n in ((0, 100), (100, 90), (250, 20)):
        seen = causal_mask(n, n, DEV)
        w, _, lim, _ = attend(q[a:a + n], k[a:a + n], v[a:a + n], 0.125, seen)
        assert_within(out[a:a + n], w, lim, f"rows {a}..{a + n}")
    assert torch.equal(out[:, 1], want[:, 1])
    if not (bad == -math.inf):
        assert not torch.isfinite(out[200:250, 0]).any()


def test_prompt_seen_infinite_value(ctx):
    """An infinite value that a row sees reaches it; the rows before do not see it."""
    g = gen(10)
    q, k, v = (randn(g, (300, 1, 64), BF) for _ in range(3))
    v[130, 0, 5] = math.inf
    _, out, _ = ctx.attention(q, k, v)
    assert torch.isfinite(out[:130]).all() and (out[130:, 0, 5] == math.inf).all()
    assert torch.isfinite(out[130:, 0, :5]).all() and torch.isfinite(out[130:, 0, 6:]).all()


def test_prompt_lowest_scores(ctx):
    """Scores at the type's lowest value, and scores of minus infinity."""
    low = torch.finfo(HF).min
    q = torch.zeros((4, 1, 8), dtype=HF, device=DEV)
    k = torch.zeros((4, 1, 8), dtype=HF, device=DEV)
    v = torch.arange(32, device=DEV).view(4, 1, 8).to(HF)
    q[:, :, 0], k[:3, :, 0] = 1.0, low
    _, out, _ = ctx.attention(q, k, v, scale=1.0)
    assert torch.allclose(out[2].float(), v[:3].float().mean(0), rtol=2e-3) and torch.allclose(out[3].float(), v[3].float())
    k[:3, :, 0] = -math.inf
    _, out, lse = ctx.attention(q, k, v, scale=1.0, need_lse=True)
    assert (out[:3] == 0).all() and (lse[:3] == -math.inf).all() and torch.allclose(out[3].float(), v[3].float())


def test_prompt_empty(ctx):
    e = torch.zeros((0, 2, 64), dtype=BF, device=DEV)
    _, out, lse = ctx.attention(e, e, e, need_lse=True)
    assert out.shape == (0, 2, 64) and lse.shape == (0, 2)
    q = torch.ones((3, 2, 64), dtype=BF, device=DEV)
    _, out, lse = ctx.attention(q, e, e, offsets([3]), offsets([0]), need_lse=True)
    assert (out == 0).all() and (lse == -math.inf).all()


def test_prompt_bad_offsets(opa, ctx):
    """Offsets that run past the rows, or backwards, or leave rows over, touch
    nothing outside and are told of."""
    g = gen(11)
    q, k, v = (randn(g, (100, 2, 64), BF) for _ in range(3))
    for off in ([0, 120], [0, 60, 40, 100], [0, 90], [5, 100], [0, -3, 100]):
        ctx.attention(q, k, v, torch.tensor(off, dtype=torch.int32, device=DEV))
        with pytest.raises(opa.OpattrError) as e:
            ctx.check()
        assert e.value.status == opa.E_INVALID_ARG
    ctx.check()
    check_prompt(ctx, q, k, v, [100], None, True)


# ---------------------------------------------------------------- the cache's single tokens
def fill(g, ctx, lens, kv, dim, page, dtype, spare=3):
    """A cache with sequences of the given lengths, appended in one call."""
    per = max(1, -(-max(lens + [1]) // page))
    c = ctx.cache(sum(-(-n // page) for n in lens) + spare, page, kv, dim, len(lens), per, dtype)
    k, v = (randn(g, (sum(lens), kv, dim), dtype) for _ in range(2))
    ctx.cache_append(c, torch.arange(len(lens), dtype=torch.int32, device=DEV), offsets(lens), k, v)
    ctx.check()
    return c, k, v


def check_token(ctx, c, q, k, v, lens, seqs=None, scale=None):
    _, out, lse = ctx.cache_attention(c, None if seqs is None else torch.tensor(seqs, dtype=torch.int32, device=DEV), q,
                                      scale=scale, need_lse=True)
    ctx.check()
    off = [0]
    for n in lens:
        off.append(off[-1] + n)
    for i, b in enumerate(range(len(lens)) if seqs is None else seqs):
        a, n = off[b], lens[b]
        seen = torch.ones((1, n), dtype=torch.bool, device=DEV)
        want, wl, lim, ll = attend(q[i:i + 1], k[a:a + n], v[a:a + n], q.shape[2] ** -0.5 if scale is None else scale, seen)
        assert_within(out[i:i + 1], want, lim, f"out of sequence {b} ({n} tokens)")
        assert_within(lse[i:i + 1], wl, ll, f"lse of sequence {b} ({n} tokens)")


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dim", [8, 64, 80, 128])
@pytest.mark.parametrize("page", [16, 64, 256])
@pytest.mark.parametrize("lens", [[1], [15, 16, 17], [0, 300, 1, 129, 64], [1500, 7]])
def test_token_lengths(ctx, dtype, dim, page, lens):
    g = gen(sum(lens) + dim + page)
    c, k, v = fill(g, ctx, lens, 2, dim, page, dtype)
    check_token(ctx, c, randn(g, (len(lens), 6, dim), dtype), k, v, lens)


@pytest.mark.parametrize("heads,kv", [(1, 1), (5, 5), (8, 1), (9, 1), (16, 2), (17, 1), (71, 1), (40, 8), (32, 2)])
@pytest.mark.parametrize("dim", [64, 128])
def test_token_heads(ctx, heads, kv, dim):
    g = gen(heads + kv)
    lens = [70, 4, 333]
    c, k, v = fill(g, ctx, lens, kv, dim, 32, BF)
    check_token(ctx, c, randn(g, (3, heads, dim), BF), k, v, lens)


def test_token_long(ctx):
    """One sequence over the whole GPU, and one beside many short ones."""
    g = gen(12)
    for lens in ([40_001], [30_011] + [1 + 3 * i for i in range(60)]):
        c, k, v = fill(g, ctx, lens, 2, 128, 64, BF)
        check_token(ctx, c, randn(g, (len(lens), 8, 128), BF), k, v, lens)


def test_token_many(ctx):
    g = gen(13)
    lens = [int(x) for x in torch.randint(0, 90, (700,), generator=torch.Generator().manual_seed(4))]
    c, k, v = fill(g, ctx, lens, 3, 64, 16, HF)
    check_token(ctx, c, randn(g, (700, 3, 64), HF), k, v, lens)


def test_token_chosen_sequences(ctx):
    g = gen(14)
    lens = [100, 5, 0, 77]
    c, k, v = fill(g, ctx, lens, 2, 64, 16, BF)
    check_token(ctx, c, randn(g, (6, 4, 64), BF), k, v, lens, seqs=[3, 0, 0, 2, 1, 3])
    q = randn(g, (4, 2, 4, 64), BF).transpose(1, 2)[:, :, 0]           # strided rows
    check_token(ctx, c, q, k, v, lens, scale=-0.2)


@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_token_past_the_end(ctx, bad):
    """What a page holds past the sequence's length, or an unused page, has no influence."""
    g = gen(15)
    lens = [37, 160]
    c, k, v = fill(g, ctx, lens, 2, 64, 64, BF)
    for x in (c.k_pages, c.v_pages):
        for b, n in enumerate(lens):
            last = int(c.table[b, n // 64])
            if last >= 0:
                x[last, :, n % 64:] = bad
        x[c.refs == 0] = bad
    check_token(ctx, c, randn(g, (2, 4, 64), BF), k, v, lens)


def test_token_repeats_exactly(ctx):
    """The same call gives the same bits, however the work was split."""
    g = gen(16)
    c, k, v = fill(g, ctx, [20_000, 3, 511], 2, 128, 32, BF)
    q = randn(g, (3, 8, 128), BF)
    first = ctx.cache_attention(c, None, q)[1]
    for _ in range(5):
        assert torch.equal(ctx.cache_attention(c, None, q)[1], first)


def test_token_bad_state(opa, ctx):
    g = gen(17)
    c, k, v = fill(g, ctx, [50, 40], 1, 64, 16, BF)
    q = randn(g, (2, 1, 64), BF)
    good = ctx.cache_attention(c, None, q)[1]
    for what, at, value in (("table", (0, 1), 10_000), ("table", (0, 2), -1), ("length", (0,), 100_000), ("length", (0,), -4)):
        t = getattr(c, what)
        old = t[at].clone()
        t[at] = value
        out = ctx.cache_attention(c, None, q)[1]
        with pytest.raises(opa.OpattrError) as e:
            ctx.check()
        assert e.value.status == opa.E_INVALID_ARG
        assert torch.equal(out[1], good[1]) and (what == "table" or (out[0] == 0).all())
        t[at] = old
    out = ctx.cache_attention(c, torch.tensor([1, 2], dtype=torch.int32, device=DEV), q)[1]
    with pytest.raises(opa.OpattrError):
        ctx.check()
    assert (out[1] == 0).all()


def test_another_stream(opa, ctx):
    """Calls from another stream than the context's are ordered on that one."""
    g = gen(18)
    side = torch.cuda.Stream()
    q, k, v = (randn(g, (3000, 4, 128), BF) for _ in range(3))
    want = ctx.attention(q, k, v)[1]
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        a = torch.zeros_like(q)
        for _ in range(20):
            a.add_(1)                                  # work the inputs wait for
        b = q + (a - 20)
        out = ctx.attention(b, k, v)[1]
        got = out.clone()
    side.synchronize()
    assert torch.equal(got, want)


def test_graph(opa):
    """The calls can be captured once their scratch is there."""
    g = gen(19)
    q, k, v = (randn(g, (200, 2, 64), BF) for _ in range(3))
    off = offsets([200])
    s = torch.cuda.Stream()
    with torch.cuda.stream(s), opa.Context(0, stream=s) as ctx:
        want = ctx.attention(q, k, v, off)[1]
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            got = ctx.attention(q, k, v, off)[1]
        got.zero_()
        graph.replay()
        s.synchronize()
        assert torch.equal(got, want)
        ctx.check()


@pytest.mark.parametrize("lens,heads,kv,dim", [([9000], 8, 1, 128), ([3000, 1, 12_000], 7, 1, 96), ([700, 700], 3, 3, 64),
                                               ([30_000], 16, 1, 64)])
def test_token_cuts(ctx, lens, heads, kv, dim):
    """Few pairs cut into many parts, and parts of unlike sequences in one run."""
    g = gen(sum(lens))
    c, k, v = fill(g, ctx, lens, kv, dim, 16, BF)
    check_token(ctx, c, randn(g, (len(lens), heads, dim), BF), k, v, lens)


def test_prompt_far_rows(ctx):
    """Rows so far apart that their places pass 32 bits."""
    g = gen(31)
    n, stride = 300, 1 << 23                                   # 2.5e9 elements from the first to the last
    x = torch.empty(n * stride, dtype=BF, device=DEV)
    q, k, v = (x[i * 128:].as_strided((n, 2, 64), (stride, 64, 1)) for i in range(3))
    for y in (q, k, v):
        y.copy_(randn(g, (n, 2, 64), BF))
    out = x[3 * 128:].as_strided((n, 2, 64), (stride, 64, 1))
    check_prompt(ctx, q, k, v, [100, 200], None, True, out=out)


def test_cache_past_32_bits(ctx):
    """The last pages of a pool of more than 2^32 elements: appended to, shared, read,
    and moved to its beginning."""
    g = gen(32)
    page, kv, dim = 128, 4, 128
    n_pages = (1 << 32) // (page * kv * dim) + 40
    c = ctx.cache(n_pages, page, kv, dim, 4, 8, BF)
    c.refs[:n_pages - 30] = 1
    c.low.fill_(n_pages - 30)
    lens = [300, 900, 0, 0]
    k, v = (randn(g, (1200, kv, dim), BF) for _ in range(2))
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    ctx.cache_append(c, i32(0, 1), i32(0, 300, 1200), k, v)
    ctx.cache_fork(c, i32(0), i32(2))
    more = [randn(g, (2, kv, dim), BF) for _ in range(2)]
    ctx.cache_append(c, i32(0, 2), i32(0, 1, 2), *more)
    assert int(c.table[c.table >= 0].min()) == n_pages - 30
    lens = [301, 900, 301, 0]
    rows = [torch.cat([x[:300], y[:1], x[300:], x[:300], y[1:]]) for x, y in zip((k, v), more)]
    q = randn(g, (4, 8, dim), BF)
    check_token(ctx, c, q, *rows, lens)
    c.refs[:n_pages - 30] = 0
    _, live = ctx.cache_compact(c)
    ctx.check()
    assert int(live) == 12 and int(c.table.max()) == 11
    check_token(ctx, c, q, *rows, lens)


def test_prompt_bad_offsets_of_runs(opa, ctx):
    """As above where keys are cut into equal runs."""
    g = gen(33)
    q = randn(g, (20, 2, 64), BF)
    k, v = (randn(g, (9000, 2, 64), BF) for _ in range(2))
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    for qo, ko in ((i32(0, 20), i32(0, 12_000)), (i32(0, 10, 20), i32(0, 9001, 9000)), (i32(0, 25, 20), i32(0, 10, 9000)),
                   (i32(3, 20), i32(0, 9000)), (i32(0, -7, 20), i32(0, -2, 9000)), (i32(0, 40), i32(0, 9000))):
        ctx.attention(q, k, v, qo, ko)
        with pytest.raises(opa.OpattrError) as e:
            ctx.check()
        assert e.value.status == opa.E_INVALID_ARG
    check_prompt(ctx, q, k, v, [20], [9000], True)

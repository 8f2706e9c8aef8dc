"""Large appends to a cache in 8 bits (GPU), pools and state whole against the model of its
definition: more rows than the blocks of threads of a launch take at once, and a page with
more sharers than a warp has lanes."""
import random

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from attn_util import randn  # noqa: E402
from test_cache8 import BF, HF, both, ctx, fresh, gen, i32  # noqa: E402, F401


@pytest.mark.parametrize("heads,dim,page,dtype", [(1, 16, 16, BF), (3, 64, 64, HF), (2, 128, 32, BF)])
def test_many_rows(ctx, heads, dim, page, dtype):  # noqa: F811
    """60,000 rows and more in a call: places of several rounds, of empty sequences and of some that go on."""
    rng, g, n = random.Random(dim), gen(dim), 37
    per = 4000 // page
    c, m = fresh(ctx, 70_000 // page + 3 * n, page, heads, dim, n, per)
    counts = [rng.choice([0, 1, 15, 16, rng.randint(1, 40)]) for _ in range(n)]
    seqs = rng.sample(range(n), n)
    k, v = (randn(g, (sum(counts), heads, dim), dtype, 0.25) for _ in range(2))
    both(ctx, c, m, seqs, counts, k, v)
    counts = [rng.choice([0, 1500, rng.randint(1, 3500)]) for _ in range(n)]
    while sum(counts) < 60_000:
        counts[rng.randrange(n)] = 3500
    # (blocks of sixteen of every size)
    grow = torch.exp2(torch.arange(sum(counts), device=k.device).div(37, rounding_mode="floor") % 19 - 9.0)[:, None, None]
    k, v = ((randn(g, (sum(counts), heads, dim), torch.float32) * grow).to(dtype) for _ in range(2))
    both(ctx, c, m, rng.sample(range(n), n), counts, k, v)
    ctx.check()
    m.same(c)


@pytest.mark.parametrize("page,heads,dim,dtype,n", [(64, 2, 64, BF, 80), (128, 1, 128, HF, 80), (32, 3, 32, BF, 80), (32, 1, 16, BF, 2300)])
@pytest.mark.parametrize("last", [3, 16, 17])
def test_more_sharers_than_lanes(ctx, page, heads, dim, dtype, n, last):  # noqa: F811
    """80 sequences, or 2,300, hold one page; each goes on at its own place of it in one call, and the last, which
    keeps it, behind fewer tokens than the others have."""
    rng, g = random.Random(page + last), gen(page + last)
    c, m = fresh(ctx, 3 * n, page, heads, dim, n, 3)
    k, v = (randn(g, (page, heads, dim), dtype) for _ in range(2))
    both(ctx, c, m, [0], [page], k, v)
    ctx.cache_fork(c, i32([0] * (n - 1)), i32(range(1, n)))
    m.fork([0] * (n - 1), range(1, n))
    order = rng.sample(range(n), n)
    to = [rng.randint(last, page - 1) for _ in range(n)]
    to[order[0]], to[order[-1]] = page - 1, last
    ctx.cache_trim(c, i32(order), i32([to[s] for s in order]))
    m.trim(order, [to[s] for s in order])
    counts = [rng.choice([1, 1, 5, 16, page]) for _ in range(n)]
    k, v = (randn(g, (sum(counts), heads, dim), dtype, 2.0 ** rng.randint(-3, 3)) for _ in range(2))
    both(ctx, c, m, order, counts, k, v)
    ctx.check()
    m.same(c)

"""Compaction of a cache whose counts of holders are not consistent (GPU)."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

DEV = "cuda:0"


@pytest.mark.parametrize("n_pages", [40, 9000])
def test_compact_with_counts_below_zero(n_pages):
    """A page with a count below 0 is as free as one with 0: pages move within the pool."""
    import paper_2609_11938_gb300 as opa
    with opa.Context(0) as ctx:
        c = ctx.cache(n_pages, 16, 1, 8, 1, n_pages)
        x = torch.arange(n_pages, device=DEV).to(torch.bfloat16)[:, None, None, None].expand_as(c.k_pages)
        c.k_pages.copy_(x)
        c.v_pages.copy_(-x)
        c.refs[::2] = 1
        c.refs[1::4] = -3
        last = (n_pages - 1) // 2 * 2
        c.table[0, 0] = last
        c.length[0] = 16
        _, live = ctx.cache_compact(c)
        ctx.check()
    moved = list(range((n_pages // 2 + 1) // 2 * 2, n_pages, 2))
    holes = list(range(1, n_pages // 2, 2))
    assert int(live) == n_pages // 2 and len(moved) == len(holes)
    want = x.clone()
    want[holes] = x[moved]
    assert torch.equal(c.k_pages, want) and torch.equal(c.v_pages, -want)
    refs = c.refs.tolist()
    assert all(r == 1 for r in refs[:n_pages // 2]) and all(r <= 0 for r in refs[n_pages // 2:])
    assert int(c.table[0, 0]) == holes[-1] and int(c.low) == n_pages // 2

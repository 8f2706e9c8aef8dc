"""Trimming the cache to lengths that are its own (GPU)."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

DEV = "cuda:0"


@pytest.mark.parametrize("per", [16, 5000])
@pytest.mark.parametrize("n", [2, 4, 900])
def test_trim_to_the_lengths_of_others(n, per):
    """Every sequence is cut to the length that the one before it has before the call."""
    import paper_2609_11938_gb300 as opa
    lens = [1 + (s * 200) // n for s in range(n)]
    offsets = [0] + torch.tensor(lens).cumsum(0).tolist()
    i32 = lambda x: torch.tensor(list(x), dtype=torch.int32, device=DEV)  # noqa: E731
    pages = [-(-x // 16) for x in lens]
    with opa.Context(0) as ctx:
        c = ctx.cache(sum(pages) + 3, 16, 1, 8, n, per)
        x = torch.zeros((offsets[-1], 1, 8), dtype=torch.bfloat16, device=DEV)
        ctx.cache_append(c, i32(range(n)), i32(offsets), x, x)
        ctx.check()
        before = c.table.clone()
        ctx.cache_trim(c, i32(range(1, n)), c.length[:n - 1])
        ctx.check()
    want = lens[:1] + lens[:-1]
    assert c.length.tolist() == want
    refs = torch.zeros_like(c.refs)
    for s, length in enumerate(want):
        held = -(-length // 16)
        assert torch.equal(c.table[s, :held], before[s, :held]) and bool((c.table[s, held:] == -1).all())
        refs[before[s, :held].long()] = 1
    assert torch.equal(c.refs, refs)
    assert bool((refs[:int(c.low)] == 1).all())

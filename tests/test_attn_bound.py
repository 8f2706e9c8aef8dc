"""The bounds of attn_bound.py tell wrong results from right ones (CPU)."""
import pytest

torch = pytest.importorskip("torch")
from attn_bound import LEAST_TOP, bound, misses  # noqa: E402
from attn_util import randn  # noqa: E402


def rounded(q, k, v, scale, keys=slice(None)):
    """Attention over some keys with the roundings that the bounds allow: weights that stand at
    LEAST_TOP rounded to the type, 32-bit sums, the result rounded once."""
    s = torch.einsum("nhd,mhd->nhm", q.float(), k[keys].float()) * scale
    w = torch.exp(s - s.amax(-1, keepdim=True)) * LEAST_TOP[q.dtype]
    o = torch.einsum("nhm,mhd->nhd", w.to(q.dtype).float(), v[keys].float())
    return (o / w.sum(-1)[..., None]).to(q.dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("m,dim", [(300, 64), (1500, 128), (9001, 128), (20_000, 64), (40_001, 128)])
def test_wrong_results_are_told(dtype, m, dim):
    g = torch.Generator()
    g.manual_seed(m)
    q = randn(g, (3, 2, dim), dtype)
    k, v = (randn(g, (m, 2, dim), dtype) for _ in range(2))
    scale = dim ** -0.5
    want, lim, rms = bound(q, k, v, scale, torch.ones((3, m), dtype=torch.bool))
    good = rounded(q, k, v, scale)
    assert misses(good, want, lim, rms) is None
    assert misses(want.to(dtype), want, lim, rms) is None
    tile = torch.cat([torch.arange(m // 2), torch.arange(m // 2 + 128, m)])
    swapped = good.clone()
    swapped[0], swapped[1] = good[1], good[0]
    for what, bad in (("zeros", torch.zeros_like(good)), ("negated", -good), ("a tile left out", rounded(q, k, v, scale, tile)),
                      ("the last tile left out", rounded(q, k, v, scale, slice(0, m - 128))), ("rows swapped", swapped),
                      ("a few percent too large", (good.float() * (1.03 if dtype == torch.bfloat16 else 1.01)).to(dtype)),
                      ("not a number", good * float("nan"))):
        assert misses(bad, want, lim, rms), what

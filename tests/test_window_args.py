"""What the calls with a window, and with a cache in 8 bits, refuse before any launch; what the
binding makes of such a cache; the definition's own pieces.  CPU only: no call here touches a GPU."""
import ctypes

import numpy as np
import pytest

torch = pytest.importorskip("torch")
import paper_2609_11938_gb300 as opa  # noqa: E402
from window_util import VALUES, codes_of, near_mask, scale_for  # noqa: E402

E4 = torch.float8_e4m3fn


class Host(opa.Context):
    """A context's argument checks on host tensors (device -1), without a GPU."""

    def __init__(self):
        self.device, self.handle, self._dev = -1, None, torch.device("cpu")

    def _enter(self):
        raise AssertionError("past the checks")


@pytest.fixture()
def host():
    return Host()


def x(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype)


def off(*v):
    return torch.tensor(v, dtype=torch.int32)


def test_struct_layouts():
    assert ctypes.sizeof(opa.Cache8) == ctypes.sizeof(opa.Cache) + 2 * 8 + 2 * 4
    assert opa.Cache8.k_scales.offset == ctypes.sizeof(opa.Cache)


def test_calls_without_a_context():
    lib, by = opa.library(), ctypes.byref
    c, r = opa.Cache8(), opa.Rows()
    assert lib.opattr_attention_window(None, by(opa.Prompt()), 4, 0) == opa.E_INVALID_ARG
    assert lib.opattr_cache_attention_window(None, by(c), None, 1, 1, by(r), by(r), None, 1.0, 4, 0) == opa.E_INVALID_ARG


@pytest.mark.parametrize("kw", [dict(window=0), dict(window=-1), dict(window=2 ** 31), dict(window=4, sinks=-1), dict(window=4, sinks=2 ** 31),
                                dict(sinks=4), dict(window=None, sinks=1)])
def test_windows(host, kw):
    with pytest.raises(ValueError, match="window|sinks"):
        host.attention(x(4, 2, 64), x(4, 2, 64), x(4, 2, 64), **kw)
    for dtype in (None, E4):
        with pytest.raises(ValueError, match="window|sinks"):
            host.cache_attention(host.cache(4, 16, 2, 64, 3, 2, dtype), None, x(2, 2, 64), **kw)


def test_window_needs_causal(host):
    with pytest.raises(ValueError, match="causal"):
        host.attention(x(4, 2, 64), x(4, 2, 64), x(4, 2, 64), off(0, 4), causal=False, window=3)
    for kw in (dict(window=3), dict(window=2 ** 31 - 1, sinks=2 ** 31 - 1)):
        with pytest.raises(AssertionError, match="past the checks"):
            host.attention(x(4, 2, 64), x(4, 2, 64), x(4, 2, 64), off(0, 4), **kw)


@pytest.mark.parametrize("dim", [8, 24, 40, 72, 120, 136, 144])
def test_dims_of_8_bits(host, dim):
    with pytest.raises(ValueError, match="head_dim"):
        host.cache(4, 16, 2, dim, 3, 2, E4)


def test_cache_of_8_bits(host):
    c = host.cache(4, 32, 2, 48, 3, 2, E4)
    assert c.k_scales.shape == (4, 2, 2) and c.struct.dtype == 2 and c.struct.k_scales == c.k_scales.data_ptr()
    rest = (c.table, c.length, c.refs, c.low)
    opa.KVCache(c.k_pages, c.v_pages, *rest, k_scales=c.k_scales, v_scales=c.v_scales)
    for scales in ((), (c.k_scales,), (None, c.v_scales), (c.k_scales[:3], c.v_scales[:3]), (c.k_scales, c.v_scales[:, :, :1])):
        with pytest.raises(ValueError, match="scales"):
            opa.KVCache(c.k_pages, c.v_pages, *rest, *scales)
    with pytest.raises(ValueError, match="scales"):
        opa.KVCache(c.k_pages.bfloat16(), c.v_pages.bfloat16(), *rest, c.k_scales, c.v_scales)
    with pytest.raises(TypeError, match="scales"):
        opa.KVCache(c.k_pages, c.v_pages, *rest, c.k_scales.double(), c.v_scales.double())
    with pytest.raises(TypeError):
        opa.KVCache(c.k_pages, c.v_pages.bfloat16(), *rest, c.k_scales, c.v_scales)
    with pytest.raises(TypeError):
        host.cache(4, 32, 2, 48, 3, 2, torch.float8_e5m2)


def test_replaced_scales(host):
    c = host.cache(4, 32, 2, 48, 3, 2, E4)
    new = c.k_scales.clone()
    c.k_scales = new
    assert c.struct.k_scales == new.data_ptr() and c.by_ref._obj is c.struct
    assert all(r._obj.k_scales == new.data_ptr() for r in c.for_rows.values())
    for wrong in (None, new[:2], new.double()):
        with pytest.raises((ValueError, TypeError)):
            c.k_scales = wrong
        assert c.k_scales is new and c.struct.k_scales == new.data_ptr()


def test_rows_of_either_type(host):
    c = host.cache(4, 16, 2, 64, 3, 2, E4)
    for dtype in (torch.bfloat16, torch.float16):
        with pytest.raises(AssertionError, match="past the checks"):
            host.cache_attention(c, None, x(2, 4, 64, dtype=dtype))
        with pytest.raises(AssertionError, match="past the checks"):
            host.cache_append(c, off(0), off(0, 1), x(1, 2, 64, dtype=dtype), x(1, 2, 64, dtype=dtype))
    assert [c.for_rows[t]._obj.rows for t in (torch.bfloat16, torch.float16)] == [0, 1]
    for dtype in (torch.float32, E4):
        with pytest.raises(TypeError):
            host.cache_attention(c, None, x(2, 4, 64, dtype=torch.float32).to(dtype))
        with pytest.raises(TypeError):
            host.cache_append(c, off(0), off(0, 1), x(1, 2, 64).to(dtype), x(1, 2, 64).to(dtype))
    with pytest.raises(TypeError):
        host.cache_append(c, off(0), off(0, 1), x(1, 2, 64), x(1, 2, 64, dtype=torch.float16))
    with pytest.raises(TypeError):
        host.cache_attention(c, None, x(2, 4, 64), out=x(2, 4, 64, dtype=torch.float16))


def test_gradients_are_not_lost_in_silence(host):
    q = x(4, 2, 64).requires_grad_()
    with pytest.raises(ValueError, match="requires a gradient"):
        host.attention(q, x(4, 2, 64), x(4, 2, 64), off(0, 4), window=3)
    c = host.cache(4, 16, 2, 64, 3, 2, E4)
    with pytest.raises(ValueError, match="requires a gradient"):
        host.cache_attention(c, off(0, 1, 2, 0), q, window=3)
    with pytest.raises(ValueError, match="requires a gradient"):
        host.cache_append(c, off(0), off(0, 4), q, q)


def test_codes():
    """The table of codes is the type's own, and the search rounds as the type does."""
    all_codes = torch.arange(256, dtype=torch.uint8)
    assert np.array_equal(all_codes.view(E4).float().numpy(), VALUES.astype(np.float32), equal_nan=True)
    v = torch.cat([torch.randn(4000) * s for s in (1e-3, 0.05, 1.0, 30.0)]).clamp(-448, 448)
    mid = torch.from_numpy((VALUES[:126] + VALUES[1:127]) / 2).float()
    v = torch.cat([v, mid, -mid, torch.tensor([448.0, -0.0, 464.0 - 16.0])])
    assert np.array_equal(codes_of(v.numpy()), v.to(E4).view(torch.uint8).numpy())
    assert codes_of([np.inf, -np.inf, np.nan, 1e9, -1e9]).tolist() == [127, 255, 127, 126, 254]


@pytest.mark.parametrize("top,e", [(0.0, -126), (448.0, 0), (448.5, 1), (1.75, -8), (2.0, -7), (3.38e38, 119), (1e-40, -126), (7.0, -6), (7.01, -5)])
def test_scales(top, e):
    assert scale_for(top) == 2.0 ** e


def test_mask():
    assert near_mask(3, 5, 2, 1, "cpu").int().tolist() == [[1, 1, 1, 0, 0], [1, 0, 1, 1, 0], [1, 0, 0, 1, 1]]
    assert near_mask(3, 2, 1, 0, "cpu").int().tolist() == [[0, 0], [1, 0], [0, 1]]

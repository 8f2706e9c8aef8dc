"""What the attention operators and the cache's calls refuse before any launch.
CPU only: no call here touches a GPU."""
import ctypes

import pytest

torch = pytest.importorskip("torch")
import paper_2609_11938_gb300 as opa  # noqa: E402


class Host(opa.Context):
    """A context's argument checks on host tensors (device -1), without a GPU."""

    def __init__(self):
        self.device, self.handle, self._dev = -1, None, torch.device("cpu")

    def _enter(self):
        raise AssertionError("a call that should have been refused")


@pytest.fixture()
def host():
    return Host()


def test_struct_layouts():
    assert ctypes.sizeof(opa.Rows) == 24
    assert ctypes.sizeof(opa.Prompt) == 8 * 4 + 2 * 8 + 4 * 24 + 3 * 8
    assert ctypes.sizeof(opa.Cache) == 6 * 4 + 8 + 6 * 8


def test_calls_without_a_context():
    lib, by = opa.library(), ctypes.byref
    c, r = opa.Cache(), opa.Rows()
    bad = opa.E_INVALID_ARG
    assert lib.opattr_attention(None, by(opa.Prompt())) == bad
    assert lib.opattr_cache_attention(None, by(c), None, 1, 1, by(r), by(r), None, 1.0) == bad
    assert lib.opattr_cache_append(None, by(c), None, 1, None, 1, by(r), by(r)) == bad
    assert lib.opattr_cache_fork(None, by(c), None, None, 1) == bad
    assert lib.opattr_cache_trim(None, by(c), None, None, 1) == bad
    assert lib.opattr_cache_compact(None, by(c), None) == bad
    assert lib.opattr_check(None) == bad
    assert opa.opattr_status_string(opa.E_PAGES) == "no free page left in the cache"


def x(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype)


def off(*v, dtype=torch.int32):
    return torch.tensor(v, dtype=dtype)


@pytest.mark.parametrize("error,q,k,v,kw", [
    (TypeError, x(4, 2, 64, dtype=torch.float32), x(4, 2, 64, dtype=torch.float32), x(4, 2, 64, dtype=torch.float32), {}),
    (TypeError, x(4, 2, 64), x(4, 2, 64, dtype=torch.float16), x(4, 2, 64), {}),
    (ValueError, x(4, 128), x(4, 2, 64), x(4, 2, 64), {}),
    (ValueError, x(4, 2, 60), x(4, 2, 60), x(4, 2, 60), {}),
    (ValueError, x(4, 2, 136), x(4, 2, 136), x(4, 2, 136), {}),
    (ValueError, x(4, 3, 64), x(4, 2, 64), x(4, 2, 64), {}),
    (ValueError, x(4, 2, 64), x(4, 2, 64), x(5, 2, 64), {}),
    (ValueError, x(4, 2, 64), x(4, 2, 64), x(4, 1, 64), {}),
    (ValueError, x(4, 2, 64), x(4, 2, 72), x(4, 2, 72), {}),
    (ValueError, x(4, 2, 128)[:, :, ::2], x(4, 2, 64), x(4, 2, 64), {}),
    (ValueError, x(4 * 2 * 68).as_strided((4, 2, 64), (136, 68, 1)), x(4, 2, 64), x(4, 2, 64), {}),
    (ValueError, x(8 * 64 + 1)[1:].view(4, 2, 64), x(4, 2, 64), x(4, 2, 64), {}),
    (ValueError, x(4, 2, 64), x(6, 2, 64), x(6, 2, 64), dict(q_offsets=off(0, 4))),
    (ValueError, x(4, 2, 64), x(4, 2, 64), x(4, 2, 64), dict(k_offsets=off(0, 4))),
    (ValueError, x(4, 2, 64), x(4, 2, 64), x(4, 2, 64), dict(q_offsets=off(0, 4), k_offsets=off(0, 2, 4))),
    (TypeError, x(4, 2, 64), x(4, 2, 64), x(4, 2, 64), dict(q_offsets=off(0, 4, dtype=torch.int64))),
    (ValueError, x(4, 2, 64), x(4, 2, 64), x(4, 2, 64), dict(q_offsets=off(0, 9, 4)[::2])),
    (ValueError, x(4, 2, 64), x(4, 2, 64), x(4, 2, 64), dict(q_offsets=off(0, 4), out=x(4, 2, 72))),
    (ValueError, x(4, 2, 64), x(4, 2, 64), x(4, 2, 64), dict(q_offsets=off(0, 4), out=x(1, 2, 64).expand(4, 2, 64))),
    (TypeError, x(4, 2, 64), x(4, 2, 64), x(4, 2, 64), dict(q_offsets=off(0, 4), out=x(4, 2, 64, dtype=torch.float16))),
])
def test_attention_refusals(host, error, q, k, v, kw):
    with pytest.raises(error):
        host.attention(q, k, v, **kw)


def test_device_is_checked():
    h = Host()
    h.device = 0
    with pytest.raises(ValueError, match="cuda:0"):
        h.attention(x(4, 2, 64), x(4, 2, 64), x(4, 2, 64))


@pytest.mark.parametrize("kw", [dict(page_size=8), dict(page_size=48), dict(page_size=2048), dict(head_dim=12),
                                dict(head_dim=256), dict(n_pages=0), dict(n_seqs=0)])
def test_cache_shapes(host, kw):
    with pytest.raises(ValueError):
        host.cache(**dict(dict(n_pages=4, page_size=16, kv_heads=2, head_dim=64, n_seqs=3, pages_per_seq=2), **kw))


def test_cache_refusals(host):
    c = host.cache(4, 16, 2, 64, 3, 2)
    with pytest.raises(TypeError):
        host.cache(4, 16, 2, 64, 3, 2, dtype=torch.float32)
    with pytest.raises(ValueError):
        opa.KVCache(c.k_pages, c.v_pages[:3], c.table, c.length, c.refs, c.low)
    with pytest.raises(ValueError):
        opa.KVCache(c.k_pages, c.v_pages, c.table, c.length[:2], c.refs, c.low)
    with pytest.raises(TypeError):
        opa.KVCache(c.k_pages, c.v_pages, c.table.long(), c.length, c.refs, c.low)
    with pytest.raises(ValueError):
        opa.KVCache(c.k_pages.transpose(1, 2).contiguous().transpose(1, 2), c.v_pages, c.table, c.length, c.refs, c.low)
    for q, seqs in ((x(2, 3, 64), None), (x(4, 2, 64), None), (x(2, 2, 72), None), (x(2, 2, 64), off(0)), (x(2, 64), None)):
        with pytest.raises(ValueError):
            host.cache_attention(c, seqs, q)
    with pytest.raises(TypeError):
        host.cache_attention(c, None, x(2, 2, 64, dtype=torch.float16))
    for args in ((off(0), off(0, 1), x(1, 2, 64), x(2, 2, 64)), (off(0), off(0), x(1, 2, 64), x(1, 2, 64)),
                 (off(0), off(0, 1), x(1, 1, 64), x(1, 1, 64))):
        with pytest.raises(ValueError):
            host.cache_append(c, *args)
    with pytest.raises(ValueError):
        host.cache_fork(c, off(0, 1), off(2))
    with pytest.raises(ValueError):
        host.cache_trim(c, off(0), off(1, 2))
    with pytest.raises(TypeError):
        host.cache_trim(c, off(0, dtype=torch.int64))

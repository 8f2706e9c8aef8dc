"""Every call of a context on prompts and caches goes through the module's function of that
name, with the arguments that the C ABI takes.  CPU only: the functions are stand-ins."""
import ctypes

import pytest

torch = pytest.importorskip("torch")
import paper_2609_11938_gb300 as opa  # noqa: E402


class Host(opa.Context):
    """A context's argument checks on host tensors (device -1), without a GPU."""

    def __init__(self):
        self.device, self.handle, self._dev = -1, None, torch.device("cpu")

    def _enter(self):
        return None


CALLS = ["opattr_attention", "opattr_attention_window", "opattr_cache_attention", "opattr_cache_attention_window",
         "opattr_cache_append", "opattr_cache_fork", "opattr_cache_trim", "opattr_cache_compact"]


@pytest.fixture()
def seen(monkeypatch):
    got = []
    for name in CALLS:
        monkeypatch.setattr(opa, name, lambda *args, name=name: got.append((name, args)) or 0)
    return got


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float8_e4m3fn])
def test_calls(seen, dtype):
    ctx, i32 = Host(), lambda *v: torch.tensor(v, dtype=torch.int32)
    c = ctx.cache(6, 16, 2, 64, 3, 2, dtype)
    x = lambda n, h: torch.zeros((n, h, 64), dtype=torch.bfloat16)  # noqa: E731
    ctx.attention(x(4, 2), x(4, 2), x(4, 2), i32(0, 4))
    ctx.attention(x(4, 2), x(4, 2), x(4, 2), i32(0, 4), window=3, sinks=1)
    ctx.cache_attention(c, i32(2, 0), x(2, 4))
    ctx.cache_attention(c, i32(2, 0), x(2, 4), window=5, sinks=2)
    ctx.cache_append(c, i32(0, 1), i32(0, 2, 3), x(3, 2), x(3, 2))
    ctx.cache_fork(c, i32(0), i32(2))
    ctx.cache_trim(c, i32(2))
    ctx.cache_compact(c)
    assert [name for name, _ in seen] == CALLS
    lib = opa.library()
    for name, args in seen:
        assert args[0] is None and len(args) == len(getattr(lib, name).argtypes)
        for given, kind in zip(args[1:], getattr(lib, name).argtypes[1:]):
            kind.from_param(given) if kind is ctypes.c_void_p else kind(given)
    assert seen[1][1][-2:] == (3, 1) and seen[3][1][-2:] == (5, 2)
    assert opa.Prompt.from_buffer_copy(seen[1][1][1]).n_seqs == 1

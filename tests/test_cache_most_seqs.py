"""Calls on the cache with numbers of sequences near 2^31 (GPU): refused on the host, before anything is launched."""
import ctypes

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("eight", [False, True])
def test_most_sequences(eight):
    import paper_2609_11938_gb300 as opa
    some = torch.zeros(4096, dtype=torch.uint8, device="cuda:0")
    p = some.data_ptr()
    with opa.Context(0) as ctx:
        c = (opa.Cache8 if eight else opa.Cache)(2 if eight else 0, 16, 1, 16, 2 ** 31 - 1, 1, 1, p, p, p, p, p, p)
        if eight:
            c.k_scales = c.v_scales = p
        rows = opa.Rows(p, 16, 16)
        by = ctypes.byref
        for n in (2 ** 31 - 1, 2 ** 31 - 1024):
            assert opa.opattr_cache_append(ctx.handle, by(c), p, n, p, 0, by(rows), by(rows)) == opa.E_INVALID_ARG
            assert opa.opattr_cache_fork(ctx.handle, by(c), p, p, n) == opa.E_INVALID_ARG
            assert opa.opattr_cache_trim(ctx.handle, by(c), p, None, n) == opa.E_INVALID_ARG
            assert opa.opattr_cache_attention(ctx.handle, by(c), p, n, 1, by(rows), by(rows), None, 1.0) == opa.E_INVALID_ARG
            assert opa.opattr_cache_attention_window(ctx.handle, by(c), p, n, 1, by(rows), by(rows), None, 1.0, 1, 0) == opa.E_INVALID_ARG
        ctx.check()

"""The serving loop of examples/attention_profile.py through a window and over a cache in 8 bits
(GPU): what its calls compute, and the traffic that it knows."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from attn_util import assert_within, attend  # noqa: E402
from window_util import attend8, near_mask, stands_for  # noqa: E402

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("attention_profile",
                                                  os.path.join(os.path.dirname(HERE), "examples", "attention_profile.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("window,sinks,eight_bits", [(None, 0, True), (20, 3, True), (20, 3, False), (500, 0, False)])
def test_loop(example, window, sinks, eight_bits):
    import paper_2609_11938_gb300 as opa
    with opa.Context(0) as ctx:
        cache, live, q, out = example.serve(example.Recorder(ctx), prompts=(40, 16, 75), steps=3, window=window, sinks=sinks,
                                            eight_bits=eight_bits)
    lengths = cache.length.tolist()
    assert [lengths[s] for s in live] == [40 + 3 + 2, 75 + 3 + 2, 40 + 3 + 2]
    for i, s in enumerate(live):
        k, v = stands_for(cache, s)
        seen = near_mask(1, lengths[s], window or lengths[s], sinks, q.device)
        if eight_bits:
            want, _, lim, _ = attend8(q[i:i + 1], k, v, example.DIM ** -0.5, seen)
        else:
            want, _, lim, _ = attend(q[i:i + 1], k, v, example.DIM ** -0.5, seen)
        assert_within(out[i:i + 1], want, lim, f"sequence {s}")


def test_profile(example, tmp_path):
    import paper_2609_11938_gb300 as opa
    rolled, matched, totals = example.main(str(tmp_path / "profile.json"), window=64, sinks=4, eight_bits=True)
    assert totals["attributed_kernels"] == totals["kernels"] == matched["direct"]
    assert (rolled["kernel_count"] > 0).all()
    n = sum((128, 70, 200, 33)) + 8 * 4 + 6 + 4          # prompts, steps, the forks' step, the last one
    held = 2 * (example.HEADS * example.DIM + example.HEADS * 4 // opa.SCALE_TOKENS)
    assert rolled["agg"][example.READ, 1] == 2 * example.ROW * n
    assert rolled["agg"][example.WRITTEN, 1] == pytest.approx(held * n, rel=1e-6)

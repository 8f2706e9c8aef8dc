"""The serving loop of examples/attention_profile.py (GPU): what its calls compute,
and what the join makes of their launches."""
import importlib.util
import json
import os

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from attn_util import assert_within, attend  # noqa: E402

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("attention_profile",
                                                  os.path.join(os.path.dirname(HERE), "examples", "attention_profile.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_loop_computes_attention(example):
    import paper_2609_11938_gb300 as opa
    with opa.Context(0) as ctx:
        cache, live, q, out = example.serve(example.Recorder(ctx), prompts=(40, 16, 75), steps=3)
    lengths = cache.length.tolist()
    assert [lengths[s] for s in live] == [40 + 3 + 2, 75 + 3 + 2, 40 + 3 + 2]
    assert sum(lengths) == sum(lengths[s] for s in live)
    # the fork shares full pages, and nothing else is left in use
    assert cache.refs.sum() == (cache.table >= 0).sum() and (cache.refs > 0).sum() == int(cache.low)
    for i, s in enumerate(live):
        rows = [x[cache.table[s][cache.table[s] >= 0].long()].transpose(1, 2).reshape(-1, example.HEADS, example.DIM)[:lengths[s]]
                for x in (cache.k_pages, cache.v_pages)]
        seen = torch.ones((1, lengths[s]), dtype=torch.bool, device=q.device)
        want, _, lim, _ = attend(q[i:i + 1], rows[0], rows[1], example.DIM ** -0.5, seen)
        assert_within(out[i:i + 1], want, lim, f"sequence {s}")


def test_profile(example, tmp_path):
    path = tmp_path / "profile.json"
    rolled, matched, totals = example.main(str(path))
    assert totals["attributed_kernels"] == totals["kernels"] == matched["direct"]
    assert totals["unattributed_ns"] == 0
    assert (rolled["kernel_count"] > 0).all()
    n = sum((128, 70, 200, 33))
    assert rolled["agg"][example.READ, 0] == 3 * example.ROW * n and rolled["agg"][example.WRITTEN, 0] == example.ROW * n
    # sums of the known traffic over the launches of an operator
    np.testing.assert_allclose(rolled["agg"][example.TIME], rolled["total_duration_ns"], rtol=1e-6)
    doc = json.loads(path.read_text())
    assert {o["operator_name"] for o in doc["operators"]} == set(example.OPERATORS)
    assert not doc["unattributed_kernels"]

"""The measured node on the GPU: a tuner and a node with real cache and
attention work, window by window."""
import pytest

from agft_workloads import get_workload
from gpu_helpers import say
from paper_2508_01744_amd import serving

pytestmark = pytest.mark.gpu


def test_tuner_runs_a_measured_node():
    out = serving.run(windows=60, layers=1, rows=16, row_tokens=512, tokens=256, heads=2, group=4, dim=64)
    say(out)
    assert out["windows"] == 60 and out["tokens"] > 0 and out["served"] > 0
    assert out["window_ms_median"] > 0 and 0 <= out["pages_used"] <= 1
    assert sum(out["arms_last_quarter"]) == 15 and len(out["arms_last_quarter"]) == get_workload(1).K


def test_pages_come_back():
    """When every request has ended, every page is free and no row holds a token."""
    node = serving.ServingNode(layers=2, rows=8, row_tokens=256, tokens=64, heads=1, group=2, dim=64, form="int8")
    batch = serving.Batch(8, 20, 64, 256, seed=1)
    for w in range(400):
        node.window(batch.window(2 if w < 20 else 0))
        assert int(node.step.counters[3]) == 0          # nothing refused
        held = (node.tables.lengths + 15) // 16
        assert int(held.sum()) + int(node.tables.counters[1]) == node.cfg.pages
        if w > 20 and batch.running == 0 and not any(batch.ended):
            break
    assert batch.served == 40 - batch.dropped and batch.running == 0
    assert int(node.tables.lengths.abs().sum()) == 0 and int(node.tables.counters[1]) == node.cfg.pages
    assert sorted(node.tables.ring.tolist()) == list(range(node.cfg.pages))

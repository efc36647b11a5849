"""The measured node's host part (CPU): continuous batching of requests."""
import numpy as np

from agft_workloads import ENV
from paper_2508_01744_amd.serving import Batch, features


def test_batches_keep_their_limits():
    """Every request's tokens come once and in order, a window never brings more
    tokens than it may, a row's pages go back exactly once per request."""
    rng = np.random.default_rng(1)
    b = Batch(rows=8, queue_cap=10, tokens=100, row_tokens=256, seed=3)
    held = [0] * 8
    asked = arrived = ends = 0
    for w in range(400):
        n = int(rng.poisson(1.0)) if w < 300 else 0
        arrived += n
        add = b.window(n)
        new = [a for a in add if a > 0]
        assert sum(new) <= 100 and len(b.queue) <= 10 and all(a >= -1 for a in add)
        for i, a in enumerate(add):
            if a == -1:
                assert held[i] > 0
                held[i] = 0
                ends += 1
            else:
                held[i] += a
                assert held[i] <= 256
        asked += sum(new)
    assert b.running == 0 and not b.queue and ends == b.served == arrived - b.dropped and asked > ends
    assert held == [0] * 8


def test_features_are_the_simulators():
    x = features(9, 0, 23, 1.0, 64, 0.54, 0.6)
    assert len(x) == 8 and x[0] == 1.0 and x[1] == 0.0 and x[3] == 0.0 and x[6] == 0.0 and x[7] == 0.0
    assert x[2] == (0.0 - ENV["mu"][1]) / ENV["sd"][1]

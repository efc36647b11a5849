"""Differential attention beside queries that are not finite."""
import pytest
import torch

from diff_reference import lambdas, weights
from gpu_helpers import say
from kv_flat import Window

pytestmark = pytest.mark.gpu
SHAPES = [(past, add, dim) for past in (3, 60, 9000) for add in (1, 5, 100) for dim in (64, 128)]


def results(past, add, dim):
    """Outputs and log sums of clean queries, and of such with a NaN in map 1 of pair 0's second head and one in map 0
    of pair 1's first, in the first and the last row."""
    say("nan", past, add, dim)
    w = Window([past, 60], [add, 1], 16, 4, 2, dim, "e4m3", "bf16", 3)
    tables, cache, step = w.on_gpu()
    lam, weight = lambdas(w, False), weights(w)
    spoilt = w.q.clone()
    spoilt[0, 3] = spoilt[w.tokens - 1, 4] = float("nan")
    o = []
    for q in (w.q, spoilt):
        lse = torch.zeros(w.tokens, 8, device="cuda")
        o.append((cache.attend_diff(tables, step, q, lam, weight=weight, lse=lse, scale=w.scale), lse))
    rows, maps = (torch.zeros(w.tokens, n, dtype=torch.bool, device="cuda") for n in (4, 8))
    rows[0, 1] = rows[w.tokens - 1, 2] = maps[0, 3] = maps[w.tokens - 1, 4] = True
    return *o, rows, maps


@pytest.mark.parametrize("past,add,dim", SHAPES)
def test_other_rows_keep_their_bits(past, add, dim):
    (out, lse), (got, got_lse), rows, maps = results(past, add, dim)
    assert bool(out.isfinite().all()) and bool(lse.isfinite().all()) and bool(got[rows].isnan().all())
    assert torch.equal(got[~rows], out[~rows]) and torch.equal(got_lse[~maps], lse[~maps])


@pytest.mark.parametrize("past,add,dim", SHAPES)
def test_log_sums_of_such_queries_are_nan(past, add, dim):
    """And not -infinity, which says that a row saw no keys."""
    _, (_, lse), _, maps = results(past, add, dim)
    assert bool(lse[maps].isnan().all())

"""A bound on a request's new tokens that the window passes: the rows that the
saved launch would have made are NaN, and the others are as ever."""
import pytest
import torch

from gpu_helpers import say
from kv_flat import Window

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("requests,group,dtype", [(6, 4, "bf16"), (70, 1, "fp16"), (1030, 2, "bf16")])
def test_a_bound_that_is_too_low(requests, group, dtype):
    say("max_new", requests, group, dtype)
    past = [30 + 7 * (i % 50) for i in range(requests)]
    add = [1 + i % 3 for i in range(requests)]
    long = [1, requests - 2]
    add[1], add[-2] = 70, 300
    w = Window(past, add, 16, 2, group, 64, "e4m3", dtype, seed=requests)
    tables, cache, step = w.on_gpu()
    shape = (w.tokens, 2 * group)
    lse, low = torch.full(shape, 7.0, device="cuda"), torch.full(shape, 7.0, device="cuda")
    right = cache.attend(tables, step, w.q, lse=lse)
    assert torch.isfinite(right).all() and torch.isfinite(lse).all()
    step.set_max_new(3)
    out = cache.attend(tables, step, w.q, out=torch.full_like(right, 7.0), lse=low)
    owner = torch.arange(requests, device="cuda").repeat_interleave(torch.tensor(add, device="cuda"))
    beyond = torch.isin(owner, torch.tensor(long, device="cuda"))
    assert torch.isnan(out[beyond]).all() and torch.isnan(low[beyond]).all()
    assert torch.equal(out[~beyond], right[~beyond]) and torch.equal(low[~beyond], lse[~beyond])
    # and a bound that holds again, over the same step
    step.set_max_new(300)
    assert torch.equal(cache.attend(tables, step, w.q), right)


def test_tokens_without_slots_beyond_the_bound():
    """Refused tokens of such a request are NaN too: nothing there is left unwritten."""
    w = Window([20, 33], [1, 90], 16, 1, 2, 128, "int8", "fp16", seed=3)
    tables, cache, step = w.on_gpu()
    tables.counters[1] = 0                                       # the pool is empty
    tables.plan(torch.tensor([1, 90], dtype=torch.int32, device="cuda"), 91, max_new=1, step=step)
    assert step.granted.tolist() == [1, 0]
    out = cache.attend(tables, step, w.q, out=torch.full_like(w.q, 7.0))
    assert torch.isfinite(out[:1]).all() and torch.isnan(out[1:]).all()

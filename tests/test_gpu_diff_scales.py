"""Differential attention of heads whose values' scales lie apart: the smaller half's
numbers, relative to themselves (diff_scales.py)."""
import pytest
import torch

from diff_scales import MOST, lambdas, smaller_half, window
from gpu_helpers import say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("form,apart", [(form, apart) for form in ("e4m3", "int8")
                                        for apart in (0, 1, 7, 12, 15, 20, 21, 22, 26, 28, 29) if apart <= MOST[form]])
def test_the_smaller_half_keeps_all_bits(form, dtype, apart):
    """Single tokens, a few rows, tiles; heads of 64 and 128 numbers; codes that lose bits first, and others."""
    for past, add, dim in (([200, 50], [1, 1], 64), ([3, 700], [1, 2], 128), ([200, 50], [70, 1], 64), ([30, 5], [150, 9], 128)):
        for codes in ("small", "large", "all"):
            say("smaller half", form, dtype, apart, past, add, dim, codes)
            w = window(past, add, dim, form, dtype, apart, codes, apart + dim)
            tables, cache, step = w.on_gpu()
            lam = lambdas(w)
            out = cache.attend_diff(tables, step, w.q, lam, gain=2.0 ** apart, scale=w.scale)
            ref, room = smaller_half(w, lam, apart)
            share = (out[..., dim:].double() - ref).abs() / room
            print("   worst share of the bound", float(share.max()), flush=True)
            assert bool((share <= 1).all()), (codes, float(share.max()), torch.nonzero(~(share <= 1))[:4].tolist())

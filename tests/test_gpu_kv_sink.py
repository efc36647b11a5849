"""One key that outweighs each of thousands of others by 2^24 and more, which
together still have their share of the output (bounds in kv_flat.py)."""
import math

import pytest
import torch

from gpu_helpers import say
from kv_flat import Window, compare

pytestmark = pytest.mark.gpu
POWERS = [23.5, 24.4, 24.9, 25.1, 27.0, 30.0]


def sink(past, new, page, heads, dim, form, dtype):
    """A request's key 0 is 1 in every number and its value 0; its other keys are
    0, with values of 0.5 to 1.9; query head g's score of key 0 is POWERS[g] in
    powers of two."""
    w = Window(past, new, page, heads, len(POWERS), dim, form, dtype, seed=5)
    w.exps[:, :, 0] = 0
    w.exps[:, :, 1] = 0 if form == "e4m3" else -6
    w.codes[:, :, 0] = 0
    first = torch.tensor([row[0] for row in w.rows], device=w.device)
    w.codes[first, :, 0, 0] = 0x38 if form == "e4m3" else 1
    w.codes[first, :, 1, 0] = 0
    size = torch.tensor(POWERS, device=w.device).repeat(heads) * math.log(2.0) / (dim * w.scale)
    w.q = size[None, :, None].expand(w.tokens, heads * len(POWERS), dim).to(w.dtype).contiguous()
    return w


@pytest.mark.parametrize("dim,form,dtype", [(64, "e4m3", "bf16"), (128, "int8", "fp16"), (256, "e4m3", "fp16")])
@pytest.mark.parametrize("new", [1, 40])
def test_one_long_context(new, dim, form, dtype):
    """131,072 tokens: one token's rows, shared out, and tiles of rows."""
    say("sink", new, dim, form, dtype)
    compare(sink([131072 - new], [new], 64, 1, dim, form, dtype), tell=(new, dim, form, dtype))


@pytest.mark.parametrize("dim,form,dtype", [(64, "e4m3", "fp16"), (128, "int8", "bf16")])
def test_single_tokens_of_many_heads(dim, form, dtype):
    """So much work that a wavefront goes over hundreds of tokens by itself."""
    say("sink", dim, form, dtype)
    compare(sink([4095] * 16, [1] * 16, 64, 16, dim, form, dtype), tell=(dim, form, dtype))

"""The bound on the half of smaller scale, on planted mistakes (in the reference, on the CPU)."""
import pytest
import torch

from diff_scales import LIFT, MOST, lambdas, smaller_half, to_fp16, window


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("form", ["e4m3", "int8"])
@pytest.mark.parametrize("add", [1, 70])
def test_the_bound_on_planted_mistakes(form, dtype, add):
    """Codes as fp16 holds them and rounded outputs pass; without the half, without the lift, or with four bits less
    of fp16's range they do not, at the last distance that keeps all bits."""
    most = MOST[form]
    for apart in (0, 12, most):
        w = window([200, 50], [add, 1], 64, form, dtype, apart, "small", apart, device="cpu")
        lam = lambdas(w)
        ref, room = smaller_half(w, lam, apart)
        power = LIFT[form] - apart
        right = smaller_half(w, lam, apart, lambda c: to_fp16(c, power))[0]
        assert torch.equal(right, ref)
        assert bool(((right.to(w.dtype).double() - ref).abs() <= room).all())
        wrong = smaller_half(w, lam, apart, lambda c: c * 0)[0]
        assert bool(((wrong - ref).abs() > room).all())
        wrong = smaller_half(w, lam, apart, lambda c: to_fp16(c, power - 4))[0]
        without = smaller_half(w, lam, apart, lambda c: to_fp16(c, -apart))[0]
        for x in (wrong, without):
            far = ((x - ref).abs() > room).double().mean()
            assert far > 0.9 if apart == most else far == 0
        # codes cut to whole multiples of 16 of their smallest step, at any distance
        step = 2.0 ** -9 if form == "e4m3" else 1.0
        wrong = smaller_half(w, lam, apart, lambda c: (c / step / 16).trunc() * 16 * step)[0]
        assert bool(((wrong - ref).abs() > room).all())


def test_a_single_bit_less_shows_too():
    for form in ("e4m3", "int8"):
        w = window([40, 9], [1, 1], 64, form, "fp16", MOST[form], "small", 1, device="cpu")
        ref, room = smaller_half(w, lambdas(w), MOST[form])
        wrong = smaller_half(w, lambdas(w), MOST[form], lambda c: to_fp16(c, LIFT[form] - MOST[form] - 1))[0]
        assert ((wrong - ref).abs() > room).double().mean() > 0.5

"""The bound of kv_flat.py on planted mistakes (CPU, in the reference): what a
right kernel may give passes, every row of a wrong sum does not."""
import pytest
import torch

from kv_flat import Window

SHAPES = [([99], "fp16"), ([31], "bf16"), ([700], "fp16"), ([150], "bf16"), ([8999], "fp16"), ([1999], "bf16")]


def window(past, dtype, form="e4m3"):
    return Window(past, [1] * len(past), 16, 1, 4, 64, form, dtype, seed=sum(past), device="cpu")


def share(got, ref, room):
    """Per row, its worst number's share of the bound."""
    return ((got - ref).abs() / room).amax(-1)


@pytest.mark.parametrize("form", ["e4m3", "int8"])
@pytest.mark.parametrize("past,dtype", SHAPES)
def test_a_rounded_reference_passes(past, dtype, form):
    w = window(past, dtype, form)
    out, lse, room, lse_room = w.reference()
    assert (share(out.to(w.dtype).double(), out, room) <= 1).all()
    rounded = w.reference(spoil=lambda p, v, past: (p / p.amax(1, keepdim=True)).half().double() * p.amax(1, keepdim=True))[0]
    assert (share(rounded.to(w.dtype).double(), out, room) <= 1).all()
    assert ((lse.float().double() - lse).abs() <= lse_room).all()
    weights = torch.exp(-lse)                                  # flat: nobody has much more than an equal share
    assert float(weights.max()) * (past[0] + 1) < 8


def spoilt(w, change):
    def spoil(p, v, past):
        change(p, v)
        return p
    got = w.reference(spoil)[0]
    ref, _, room, _ = w.reference()
    return share(got, ref, room)


def scaled(lo, hi, factor):
    def change(p, v):
        p[:, lo:hi] *= factor
    return change


@pytest.mark.parametrize("past,dtype", SHAPES[:2])
def test_a_single_key(past, dtype):
    w = window(past, dtype)
    n = past[0]
    for change in (scaled(n, n + 1, 0), scaled(0, 1, 0), scaled(n, n + 1, 2), scaled(15, 16, 0), scaled(16, 17, 0)):
        assert (spoilt(w, change) > 1).all()


@pytest.mark.parametrize("past,dtype", SHAPES)
def test_blocks_units_and_halves(past, dtype):
    w = window(past, dtype)
    n = past[0] + 1
    last = max(0, (n - 1) // 64 * 64 if n % 64 > 16 else n - 64)
    changes = [scaled(0, 64, 0), scaled(last, n, 0), scaled(0, 64, 2), scaled(0, n // 2, 0), scaled(n // 2, n, 2),
               scaled(0, n, 0), scaled(0, n, 0.98)]
    if n < 200 or dtype == "fp16" and n < 1000:
        changes += [scaled(16, 32, 0), scaled(n // 16 * 16 - 16, n // 16 * 16, 2)]
    for k, change in enumerate(changes):
        assert (spoilt(w, change) > 1).all(), k


@pytest.mark.parametrize("past,dtype", [SHAPES[0], SHAPES[3]])
def test_keys_in_each_others_places(past, dtype):
    """The weights of two blocks, or of two pages' halves, exchanged."""
    def exchange(a, b, n):
        def change(p, v):
            p[:, a:a + n], p[:, b:b + n] = p[:, b:b + n].clone(), p[:, a:a + n].clone()
        return change
    w = window(past, dtype)
    found = [(spoilt(w, exchange(a, b, 16)) > 1).double().mean() for a, b in ((0, 16), (16, 64), (32, 80))]
    assert sum(found) / 3 > 0.5


def test_logarithms_see_a_key():
    for n, dtype in ((99, "fp16"), (2999, "bf16")):
        w = window([n], dtype)
        _, lse, _, room = w.reference()
        without = torch.log(torch.exp(lse) * (1 - 0.3 / (n + 1)))     # a key of less than a third of the mean weight
        assert ((without - lse).abs() > room).all()

"""What the measured node cannot serve is refused at once (CPU)."""
import pytest

from paper_2508_01744_amd.serving import Batch, run


@pytest.mark.parametrize("kw", [dict(row_tokens=31), dict(row_tokens=7), dict(row_tokens=0), dict(rows=0), dict(tokens=0)])
def test_batches_without_room(kw):
    """Requests are drawn from 16 prompt and 4 output tokens up, within half and an
    eighth of a row: shorter rows would be asked for tokens that never fit."""
    with pytest.raises(ValueError):
        Batch(**{**dict(rows=4, queue_cap=4, tokens=64, row_tokens=256), **kw})


def test_the_shortest_rows():
    b = Batch(rows=3, queue_cap=5, tokens=20, row_tokens=32, seed=2)
    held = [0] * 3
    for w in range(200):
        for i, a in enumerate(b.window(1 if w < 100 else 0)):
            held[i] = 0 if a < 0 else held[i] + a
            assert held[i] <= 32
    assert b.running == 0 and b.served == 100 - b.dropped


@pytest.mark.parametrize("windows", [0, -3])
def test_no_windows(windows):
    with pytest.raises(ValueError, match="window"):
        run(windows=windows)

"""Attention whose every key counts, on the GPU against 64 bits, by each way that
the work is split and joined (data and bounds in kv_flat.py; that the bounds see a
key, a block, a piece too few or too much is shown in test_kv_flat_bound.py).

Few rows (a request's tokens x group up to 16, up to 64 while that is little work)
are units of 64 tokens, per head and 16 rows.  Workgroups: 1,024, 768 or 512 for
heads of 64, 128 and 256 numbers; a workgroup's share is at least 4 units, and up to
8 of them rows are cut evenly if that takes no more workgroups."""
import os
import re

import pytest
import torch

from gpu_helpers import say
from kv_flat import Window, compare

pytestmark = pytest.mark.gpu
GROUPS = {64: 1024, 128: 768, 256: 512}
COMMON = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2508_01744_amd", "csrc",
                      "agft_kv_common.h")


def constant(name):
    return int(re.search(rf"constexpr int {name} = (\d+);", open(COMMON).read()).group(1))


def planned(step):
    """Units of few rows and items of many rows, per head, that the plan wrote:
    the last work entry, behind counters, starts, granted and lengths."""
    requests = step.cfg.requests
    row = -(-(requests + 1) * 4 // 256) * 256
    at = 256 + 3 * row + 32 * requests
    return step.buffer[at:at + 8].view(torch.int32).tolist()


def units(w):
    """Units of single tokens' rows, over all heads."""
    rows = [a * w.group for a in w.add]
    assert max(rows) <= 16
    return w.heads * sum(-(-(p + a) // 64) for p, a in zip(w.past, w.add) if a > 0)


def share_of(w):
    return max(4, -(-units(w) // GROUPS[w.dim]))


@pytest.mark.parametrize("dim,group,form,dtype", [(64, 1, "e4m3", "fp16"), (64, 16, "int8", "bf16"), (128, 4, "int8", "fp16"),
                                                   (128, 3, "e4m3", "bf16"), (256, 5, "e4m3", "fp16"), (256, 8, "int8", "fp16")])
def test_single_tokens_of_every_length(dim, group, form, dtype):
    """One token over 0 to 200 held, and about units' ends beyond: whole rows in one
    workgroup, and pieces of them."""
    past = list(range(0, 201, 3)) + [255, 256, 257, 319, 320, 321, 511, 512, 513, 767, 768, 1023, 1024, 1600]
    compare(Window(past, [1] * len(past), 16, 2, group, dim, form, dtype, seed=dim + group), tell=(dim, group, form, dtype))


@pytest.mark.parametrize("page,dim,dtype", [(16, 64, "fp16"), (32, 128, "fp16"), (128, 256, "fp16"), (64, 128, "bf16")])
def test_few_rows_of_several_tokens(page, dim, dtype):
    """Drafted tokens: masks that end inside a block, a page, a unit."""
    past = [0, 1, 5, 13, 14, 15, 16, 60, 61, 62, 63, 64, 100, 126, 127, 128, 200, 333]
    add = [1 + (3 * i) % 5 for i in range(len(past))]
    compare(Window(past, add, page, 3, 3, dim, "e4m3", dtype, seed=page), tell=(page, dim, dtype))


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_even_pieces_of_long_rows(dim):
    """One request's rows in so many pieces that they are joined in two levels, and
    a few that are joined in one."""
    for past in ([40 * 4 * 64 + 17], [5 * 4 * 64 - 1, 31 * 4 * 64, 33 * 4 * 64, 900]):
        w = Window(past, [1] * len(past), 64, 1, 4, dim, "e4m3", "fp16", seed=dim)
        assert share_of(w) == 4 and max(past) // 256 >= 32
        compare(w, tell=(dim, past))


LARGE = [   # dim, heads, group, lengths: shares beyond 8, equal stretches whatever the rows
    (64, 1, 16, [600000]),                              # every workgroup in the middle of one request, 938 pieces
    (128, 2, 4, [90001, 70013, 50000]),                 # stretches over rows' ends, pieces beyond 32
    (256, 1, 8, [7000 + 31 * i for i in range(40)]),    # pieces of one level, two rows in a stretch
    (64, 8, 2, [100 + 997 * (i % 37) for i in range(70)]),      # short rows whole within a stretch beside long ones
]


@pytest.mark.parametrize("dim,heads,group,past", LARGE)
def test_equal_stretches_of_much_work(dim, heads, group, past):
    w = Window(past, [1] * len(past), 128, heads, group, dim, "int8", "fp16", seed=dim)
    assert share_of(w) > 8
    say("share", share_of(w))
    compare(w, tell=(dim, heads, len(past)))


@pytest.mark.parametrize("requests,heads,length", [(60, 12, 64 * 11), (600, 1, 64 * 9), (1000, 2, 64 * 3)])
def test_rows_that_cannot_be_cut_evenly(requests, heads, length):
    """Shares of at most 8 whose even cuts would take more workgroups than there are:
    up to 64 requests, and up to 1,024."""
    w = Window([length - 1] * requests, [1] * requests, 64, heads, 1, 64, "e4m3", "fp16", seed=requests)
    share = share_of(w)
    assert share <= 8
    for s in (share, share + 2):
        assert requests * heads * -(-length // 64 // s) > 1024
    compare(w, tell=(requests, heads))


@pytest.mark.parametrize("dim,group,dtype", [(64, 1, "fp16"), (128, 4, "fp16"), (256, 3, "fp16"), (128, 7, "bf16"), (64, 128, "fp16")])
def test_prompts_and_chunks(dim, group, dtype):
    """Tiles of 128 rows: remainders of rows and of tokens, with and without tokens held."""
    add = [-(-r // group) for r in (65, 100, 127, 128, 129, 160, 257, 400)]
    past = [0, 3, 60, 64, 65, 128, 300, 0]
    compare(Window(past, add, 32, 2, group, dim, "e4m3", dtype, seed=group), tell=(dim, group, dtype))


@pytest.mark.parametrize("dim,page,past,new", [(64, 64, 9000, 130), (128, 16, 4097, 33), (256, 128, 6000, 40), (128, 32, 20000, 70)])
def test_chunks_whose_tokens_are_shared_out(dim, page, past, new):
    """A tile's tokens in several parts."""
    w = Window([past, 10], [new, 1], page, 1, 4, dim, "int8", "fp16", seed=past)
    step = compare(w, tell=(dim, past, new))[2]
    assert planned(step)[1] > 2 * -(-new * 4 // 128)


@pytest.mark.parametrize("heads", [1, 3])
@pytest.mark.parametrize("over", [-2, 0, 1])
def test_where_tiles_begin_to_pay(heads, over):
    """Requests of 17 to 64 rows: 16 rows at a time up to a number of units per head,
    tiles beyond."""
    budget = constant("kMidUnits") // heads
    left, past, add = budget + over, [], []
    if left % 2:                                    # 48 rows over one unit
        past, add, left = [20], [6], left - 3
    while left > 0:                                 # 24 rows over up to 64 units
        n = min(64, left // 2)
        past, add, left = past + [64 * n - 3 - len(past) % 50], add + [3], left - 2 * n
    w = Window(past, add, 128, heads, 8, 64, "e4m3", "fp16", seed=heads)
    step = compare(w, tell=(heads, over))[2]
    few, items = planned(step)
    if over <= 0:
        assert (few, items) == (budget + over, 0)
    else:
        assert few == 0 and items >= len(past)


@pytest.mark.parametrize("requests", [1024, 1030])
def test_some_rows_of_many_requests(requests):
    """17 to 64 rows of each of about 1,024 requests: beyond them always tiles."""
    past = [3 + (7 * i) % 90 for i in range(requests)]
    w = Window(past, [3 + i % 6 for i in range(requests)], 16, 1, 8, 64, "int8", "fp16", seed=requests)
    step = compare(w, tell=requests)[2]
    if requests > 1024:
        assert planned(step)[0] == 0 and planned(step)[1] == requests


def test_everything_beside_everything():
    """Idle, single, drafted, chunks and a prompt in one window; more than 64 requests."""
    past = [(37 * i) % 1500 for i in range(90)]
    add = [(1, 1, 0, 2, 1, 40, 1, 3)[i % 8] for i in range(90)]
    add[11], past[11], past[50] = 500, 0, 12000
    for max_new in (500, None):
        compare(Window(past, add, 32, 2, 4, 128, "e4m3", "fp16", seed=8), max_new=max_new, tell=max_new)

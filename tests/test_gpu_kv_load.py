"""What plans, trims and compactions make of tables with pages in common, on the GPU."""
import pytest
import torch

from gpu_helpers import say
from paper_2508_01744_amd import KvTables, kv_config

pytestmark = pytest.mark.gpu


def ints(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def loaded(requests, lengths, rows, free, shared, pages=40):
    """The first requests' lengths and rows; the others hold nothing."""
    tables = KvTables(kv_config(requests, 64, pages, page=16, heads=1, group=1, dim=64))
    n, table = ints(*lengths, *[0] * (requests - len(lengths))), torch.zeros(requests, 4, dtype=torch.int32, device="cuda")
    table[:len(rows)] = ints(*sum(rows, [])).view(-1, 4)
    tables.load(n, table, ints(*free), shared=shared)
    return tables


def asked(requests, *first):
    return ints(*first, *[0] * (requests - len(first)))


@pytest.mark.parametrize("requests", [3, 70, 1025])
def test_nobody_ends_where_owners_are_not_counted(requests):
    """No page goes back, however often it is named: two later requests would have been given it."""
    say("uncounted", requests)
    rows = [[5, 6, 7, 9], [5, 6, 8, 0], [5, 9, 9, 9]]
    tables = loaded(requests, [48, 33, 16], rows, [1, 2, 3], False)
    for _ in range(2):
        step = tables.plan(asked(requests, -1, 2, -1), 8)
        assert step.counters.tolist()[:6] == [0, 3, 2, 2, 0, 0] and step.granted.tolist()[:3] == [0, 2, 0]
        assert step.slots.tolist()[:3] == [8 * 16 + 1, 8 * 16 + 2, -1] and step.lengths.tolist()[:3] == [48, 35, 16]
        edit = tables.trim(ints(0, 16, 16, *[-1] * (requests - 3)))         # (the third one has no more)
        assert edit.counters.tolist() == [0, 3, 0, 2, 0, 0, 0, 2] and edit.lengths.tolist()[:3] == [48, 33, 16]
        tables.commit(edit)
    assert tables.counters.tolist() == [0, 3, 0, 1, 0, 0, 0, 0] and tables.ring.tolist()[:3] == [1, 2, 3]
    tables.reset()
    tables.commit(tables.plan(asked(requests, 5, 5), 10))
    tables.commit(tables.plan(asked(requests, -1, -1), 1))
    assert tables.counters.tolist()[1:4] == [40, 0, 0]


@pytest.mark.parametrize("requests", [4, 1025])
def test_no_new_tokens_in_a_page_that_others_hold(requests):
    """Windows of the requests of one partly filled page are refused until one of them ends; whole pages in common do
    not matter."""
    say("partly filled", requests)
    tables = loaded(requests, [20, 27, 18, 16], [[5, 6, 9, 9], [5, 6, 9, 9], [5, 7, 9, 9], [8, 0, 9, 9]], [1, 2, 3], True)
    for stream in (None, torch.cuda.Stream()):
        tables.set_stream(stream)
        torch.cuda.synchronize()
        for add in ((1, 0, 0, 0), (0, 30, 1, 0)):
            with pytest.raises(ValueError, match="in part"):
                tables.plan(asked(requests, *add), 40)
        step = tables.plan(asked(requests, 0, -1, 3, 3), 8)
        torch.cuda.synchronize()
        assert step.counters.tolist()[:6] == [1, 2, 6, 1, 1, 0]
        assert step.slots.tolist() == [7 * 16 + 2, 7 * 16 + 3, 7 * 16 + 4, 16, 17, 18, -1, -1]
    tables.set_stream(None)
    tables.commit(step)
    graph, step = torch.cuda.CUDAGraph(), tables.plan(asked(requests, 0, 0, 1), 1)
    torch.cuda.synchronize()
    add = asked(requests, 0, 0, 1)
    with pytest.raises(ValueError, match="recorded"), torch.cuda.graph(graph):
        add.clone()
        tables.plan(add, 1, step=step)
    torch.cuda.synchronize()
    tables.commit(tables.trim(ints(0, *[-1] * (requests - 1))))
    step = tables.plan(asked(requests, 0, 30), 40)
    assert step.granted.tolist()[1] == 30 and step.slots.tolist()[0] == 6 * 16 + 11
    step, graph = tables.plan(add, 1), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        tables.plan(add, 1, step=step)
    step.slots.zero_()
    graph.replay()
    assert step.slots.tolist() == [7 * 16 + 5]

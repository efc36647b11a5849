"""Which tables KvTables.load takes over (CPU: calls that would launch are noted by
kv_stub.py instead)."""
import contextlib

import pytest
import torch

import kv_stub
from paper_2508_01744_amd import KvTables, kv_config

PAGES = 40


@pytest.fixture
def tables(monkeypatch):
    kv_stub.install(monkeypatch)
    t = KvTables(kv_config(requests=3, row_tokens=64, pages=PAGES, page=16, heads=2, group=1, dim=64))
    t._settled = contextlib.nullcontext
    return t


def ints(*x):
    return torch.tensor(x, dtype=torch.int32)


LENGTHS = ints(48, 33, 0)
TABLE = ints(5, 6, 7, 30, 8, 9, 10, 31, 5, 5, 5, 5).view(3, 4)     # (behind the tokens: what earlier ones left)


@pytest.mark.parametrize("shared", [False, True])
def test_free_pages_that_are_not(tables, shared):
    before = tables.buffer.clone()
    for free, match in ((ints(1, 2, 1), "twice"), (ints(39, 39), "twice"), (ints(1, 7), "holds"), (ints(10), "holds"),
                        (ints(5, 0), "holds")):
        with pytest.raises(ValueError, match=match):
            tables.load(LENGTHS, TABLE, free, shared=shared)
        assert torch.equal(tables.buffer, before)
    for free in (ints(1, 2, 3), ints(30, 31), ints(), ints(*[p for p in range(PAGES) if p not in (5, 6, 7, 8, 9, 10)])):
        tables.load(LENGTHS, TABLE, free, shared=shared)
        assert tables.counters.tolist()[:2] == [0, free.numel()] and tables.ring.tolist()[:free.numel()] == free.tolist()
        assert torch.equal(tables.lengths, LENGTHS) and torch.equal(tables.table, TABLE)
    tables.load(ints(0, 0, 0), TABLE, torch.arange(PAGES, dtype=torch.int32), shared=shared)


COMMON = ints(5, 6, 7, 9, 5, 6, 8, 0, 5, 9, 9, 9).view(3, 4)


def test_pages_in_common_that_nobody_counts(tables):
    """They stay whole: counters[3] tells the kernels that no page can be given back."""
    tables.load(ints(48, 33, 16), COMMON, ints(1, 2, 3))
    assert tables.counters.tolist() == [0, 3, 0, 1, 0, 0, 0, 0] and not tables.owners.any()
    tables.load(ints(48, 33, 16), COMMON, ints(1, 2, 3), shared=True)
    assert tables.counters.tolist() == [0, 3, 3, 0, 0, 0, 0, 0] and tables.owners.tolist()[5:7] == [2, 1]
    tables.load(LENGTHS, TABLE, ints(1, 2, 3))
    assert tables.counters.tolist() == [0, 3, 0, 0, 0, 0, 0, 0]
    before = tables.buffer.clone()
    for lengths in (ints(20, 33, 16), ints(48, 32, 1), ints(17, 17, 0)):
        with pytest.raises(ValueError, match="in part"):
            tables.load(lengths, COMMON, ints(1, 2, 3))
        assert torch.equal(tables.buffer, before)


def test_no_new_tokens_in_a_page_that_others_hold(tables):
    """Both would write there; once one of them is gone the other gets tokens again."""
    t = tables
    t.load(ints(20, 27, 16), COMMON, ints(1, 2, 3), shared=True)
    for add in (ints(1, 0, 0), ints(0, 5, 1), ints(1, 1, 1)):
        with pytest.raises(ValueError, match="in part"):
            t.plan(add, 8)
    for add in (ints(0, 0, 1), ints(-1, 0, 0)):
        t.plan(add, 8)
    with pytest.raises(ValueError, match="in part"):
        t.plan(ints(0, 1, 0), 8)
    t.owners[6] = 0                                     # (the kernels are not run here)
    t.lengths[0] = 0
    t.plan(ints(0, 1, 0), 8)
    assert not t._partly
    for again in (lambda: t.load(ints(48, 33, 16), COMMON, ints(1, 2, 3), shared=True), t.reset):
        t.load(ints(20, 27, 16), COMMON, ints(1, 2, 3), shared=True)
        assert t._partly
        again()
        t.plan(ints(1, 1, 1), 8)

"""Forks, trims, compaction and page copies on the GPU against pages_reference.py:
whole numbers, and copies of codes, compared exactly."""
import ctypes

import numpy as np
import pytest
import torch

from gpu_helpers import say
from pages_reference import Pages
from paper_2508_01744_amd import KvCache, KvEdit, KvTables, _lib as L, kv_config

pytestmark = pytest.mark.gpu


def make(requests, row_pages, pages, page=16, heads=2, group=1, dim=64, form="e4m3"):
    cfg = kv_config(requests, row_pages * page, pages, page=page, heads=heads, group=group, dim=dim, form=form)
    return KvTables(cfg), KvCache(cfg), Pages(requests, row_pages, pages, page, heads, group, dim, form)


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def same_tables(tables, node):
    """Everything that the tables say of pages in use and of free ones."""
    assert tables.lengths.tolist() == node.lengths
    assert tables.counters.tolist() == [node.head, node.free, node.extra, 0, 0, 0, 0, 0]
    assert tables.owners.tolist() == node.owners
    got, ring = tables.table.cpu().numpy(), tables.ring.tolist()
    for i, n in enumerate(node.lengths):
        used = node._pages(n)
        assert (got[i, :used] == node.table[i, :used]).all(), i
    free = [ring[(node.head + m) % node.P] for m in range(node.free)]
    assert free == [node.ring[(node.head + m) % node.P] for m in range(node.free)]
    held = {}
    for i, n in enumerate(node.lengths):
        for m in range(node._pages(n)):
            held[int(got[i, m])] = held.get(int(got[i, m]), 0) + 1
    assert len(free) == len(set(free)) and not set(free) & set(held) and len(free) + len(held) == node.P
    assert all(node.owners[p] == c - 1 for p, c in held.items())


def same_edit(edit, want):
    assert edit.counters.tolist() == want["counters"]
    assert edit.lengths.tolist() == want["lengths"]
    moves = edit.moves.tolist()
    if want["kind"] != "trim":
        assert moves == want["moves"] + [[-1, -1]] * (len(moves) - len(want["moves"]))
    if want["kind"] == "fork":
        assert edit.granted.tolist() == want["granted"]


class Both:
    """The package and the reference, side by side, with what each request's tokens are."""

    def __init__(self, *args, seed=0, **kw):
        self.tables, self.cache, self.node = make(*args, **kw)
        self.rng, self.held = np.random.default_rng(seed), [[] for _ in range(self.node.R)]
        self.next = 1

    def edit(self, name, *args):
        node = self.node
        tensors = [None if a is None else ints(a) for a in args]
        first = getattr(self.tables, name)(*tensors)
        before = first.counters.tolist()
        edit = getattr(self.tables, name)(*tensors, edit=first)            # planning changes no state
        assert edit is first and edit.counters.tolist() == before
        want = getattr(node, name)(*args)
        same_edit(edit, want)
        self.cache.copy(edit)
        node.copy(want)
        old = self.held
        self.held = [list(h) for h in old]
        if name == "fork":
            for a, b, g in zip(args[0], args[1], want["granted"]):
                if g:
                    self.held[b] = old[a][:g]
        self.held = [h[:n] for h, n in zip(self.held, want["lengths"])]
        self.tables.commit(edit)
        node.commit_edit(want)
        same_tables(self.tables, node)
        return want

    def window(self, add):
        """New tokens whose keys and values are numbers of their own."""
        n, node = max(1, sum(a for a in add if a > 0)), self.node
        step = self.tables.plan(ints(add), n)
        want = node.plan(add, n)
        assert step.counters.tolist() == want["counters"] and step.slots.tolist() == want["slots"]
        x = self.rng.integers(-7, 8, (2, n, node.H, node.D)).astype(np.float64)
        x[:, :, :, 0] = 7                                   # (one scale for all: stored as they are)
        k, v = (torch.tensor(z, dtype=torch.float32, device="cuda") for z in x)
        self.cache.append(step, k, v)
        node.append(want, *x)
        for i, g in enumerate(want["granted"]):
            at = want["starts"][i]
            self.held[i] = [] if want["lengths"][i] == 0 else self.held[i] + [x[:, t].astype(np.float32) for t in range(at, at + g)]
        self.tables.commit(step)
        node.commit(want)
        same_tables(self.tables, node)

    def same_tokens(self):
        """Every request's tokens read back as what was written."""
        table = self.tables.table.cpu().numpy()
        slots = [int(table[i, t // self.node.page]) * self.node.page + t % self.node.page
                 for i, n in enumerate(self.node.lengths) for t in range(n)]
        if slots:
            k, v = self.cache.export(torch.tensor(slots, device="cuda"), torch.float32)
            want = np.stack([x for h in self.held for x in h], 1)
            assert (k.cpu().numpy() == want[0]).all() and (v.cpu().numpy() == want[1]).all()
        assert [len(h) for h in self.held] == self.node.lengths


@pytest.mark.parametrize("requests,row_pages,pages,page,seed", [
    (2, 1, 3, 16, 0), (3, 5, 9, 16, 1), (7, 6, 30, 32, 2), (40, 5, 120, 16, 3), (65, 4, 200, 64, 4), (130, 7, 500, 16, 5),
    (30, 3, 33, 128, 6), (1030, 3, 1500, 16, 7), (2500, 2, 3000, 16, 8)])
def test_histories(requests, row_pages, pages, page, seed):
    """Windows, forks, trims and compactions in any order, with pools that run short."""
    say("histories", requests, row_pages, pages, page, seed)
    both = Both(requests, row_pages, pages, page, seed=seed)
    rng = both.rng
    for turn in range(14 if requests < 500 else 6):
        kind = rng.integers(0, 4)
        n = both.node.lengths
        if turn == 0 or kind == 0:
            few = rng.integers(0, 3, requests)
            add = np.select([few == 0, few == 1], [0, rng.integers(1, 2 * page, requests)], 1)
            if turn % 3 == 2:
                add[rng.integers(0, requests, 2)] = -1
            both.window(add.tolist())
        elif kind == 1:
            count = int(rng.integers(1, requests + 3))
            src = rng.integers(-1, requests + 1, count).tolist()
            dst = (rng.permutation(requests + 2)[:count] - 1).tolist()
            if count > 2:
                dst[-1] = dst[0]                            # named twice: refused both times
            tokens = None if turn % 2 else [int(rng.integers(-1, max(2, 2 * n[a] if 0 <= a < requests else 2))) for a in src]
            both.edit("fork", src, dst, tokens)
        elif kind == 2:
            keep = [int(rng.choice([-1, 0, x, x + 1, x - 1, rng.integers(0, x + 1), x // page * page])) for x in n]
            both.edit("trim", keep)
        else:
            both.edit("compact")
        if requests < 500 or turn > 3:
            both.same_tokens()


@pytest.mark.parametrize("n", [1, 1023, 1024, 1025, 2600])
def test_many_forks_at_once(n):
    """One launch's forks and two launches', one source for all, a pool that runs short."""
    say("forks", n)
    both = Both(n + 1, 3, n // 2 + 5, 16, seed=n)
    both.window([37] + [0] * n)
    order = both.rng.permutation(n) + 1
    want = both.edit("fork", [0] * n, order.tolist(), [int(x) for x in both.rng.integers(1, 40, n)])
    assert n < 9 or 0 < want["counters"][3] < n
    both.same_tokens()
    both.edit("trim", [0] * (n + 1))
    assert both.node.free == both.node.P and both.node.extra == 0
    both.window([5] * (n + 1))


@pytest.mark.parametrize("requests", [6, 1500, 4000])
def test_refused_trims_are_counted(requests):
    """One in three requests would end inside a page that others hold, wherever it stands among the requests."""
    both = Both(requests, 2, 2 * requests, 16, seed=requests)
    third = requests // 3
    both.window([17] * third + [0] * (requests - third))
    both.edit("fork", list(range(third)) * 2, list(range(third, 3 * third)), None)
    want = both.edit("trim", [int(x) for x in both.rng.choice([-1, 0, 5, 16], requests)])
    assert want["counters"][3] > requests // 8 or requests < 9
    both.same_tokens()


def test_long_rows():
    """Rows of more entries than one workgroup copies or lets go at a time; pages go back by their last owner."""
    tables, cache, node = make(6, 2600, 6000)
    node.lengths = [2599 * 16 + 3, 0, 0, 0, 0, 0]
    order = np.random.default_rng(3).permutation(6000)
    node.table[0, :2600] = order[:2600]
    node.ring = [int(x) for x in order[2600:]] + [0] * 2600
    node.free = 3400
    tables.load(ints(node.lengths), ints(node.table.tolist()), ints(node.ring[:3400]))
    for src, dst, tokens in (([0, 0, 0], [1, 2, 5], [2599 * 16 + 3, 1025 * 16, 1024 * 16 + 1]), ([1, 2], [3, 4], None)):
        edit, want = tables.fork(ints(src), ints(dst), None if tokens is None else ints(tokens)), node.fork(src, dst, tokens)
        same_edit(edit, want)
        tables.commit(edit)
        node.commit_edit(want)
        same_tables(tables, node)
    for keep in ([0, -1, 700 * 16, 0, -1, 0], [-1, 0, -1, -1, 100 * 16, -1], [0, 0, 0, 0, 0, 0]):
        edit, want = tables.trim(ints(keep)), node.trim(keep)
        same_edit(edit, want)
        tables.commit(edit)
        node.commit_edit(want)
        same_tables(tables, node)
    assert node.free == 6000


@pytest.mark.parametrize("pages", [1, 2, 31, 32, 33, 4097, (1 << 18) - 1, 1 << 18, (1 << 18) + 1, 700001])
@pytest.mark.parametrize("share", [0.0, 0.3, 1.0])
def test_compaction_of_pools(pages, share):
    """Pools of whose free bits a workgroup keeps all, and larger ones; none, some or all pages held."""
    say("compact", pages, share)
    rng = np.random.default_rng(pages)
    held = int(round(pages * share))
    width = max(1, -(-held // 3))
    cfg = kv_config(4, width * 16, pages, heads=1, group=1, dim=64)
    tables = KvTables(cfg)
    order = rng.permutation(pages).astype(np.int32)
    table, lengths = np.zeros((4, width), np.int32), np.zeros(4, np.int32)
    for i in range(3):
        part = order[:held][i * width:(i + 1) * width]
        table[i, :part.size], lengths[i] = part, 16 * part.size - (5 if part.size else 0)
    table[3, :1], lengths[3] = table[0, :1], min(16, lengths[0])            # a page of two owners
    tables.load(*(torch.tensor(x, device="cuda") for x in (lengths, table, order[held:])), shared=True)
    edit = tables.compact()
    tables.compact(edit=edit)
    free = np.zeros(pages, bool)
    free[order[held:]] = True
    src, dst = np.nonzero(~free[held:])[0] + held, np.nonzero(free[:held])[0]
    moves = np.full((max(1, pages // 2), 2), -1)
    moves[:src.size] = np.stack([src, dst], 1)
    extra = int(held > 0)
    assert (edit.moves.cpu().numpy() == moves).all()
    assert edit.counters.tolist() == [held % pages, pages - held, extra, 0, 0, 0, src.size, 3]
    to = np.arange(pages)
    to[src] = dst
    tables.commit(edit)
    got = tables.table.cpu().numpy()
    for i in range(4):
        used = -(-lengths[i] // 16)
        assert (got[i, :used] == to[table[i, :used]]).all()
    owners = tables.owners.cpu().numpy()
    assert owners.sum() == extra and (not extra or owners[to[table[0, 0]]] == 1)
    assert (tables.ring.cpu().numpy() == np.arange(pages)).all()
    assert tables.counters.tolist() == [held % pages, pages - held, extra, 0, 0, 0, 0, 0]
    assert tables.lengths.tolist() == lengths.tolist()


@pytest.mark.parametrize("heads,page,dim,form", [(1, 16, 64, "int8"), (3, 32, 128, "e4m3"), (8, 128, 256, "int8"),
                                                  (5, 16, 64, "e4m3"), (7, 64, 128, "int8")])
def test_copies_are_whole_and_touch_nothing_else(heads, page, dim, form):
    """All codes, whatever they stand for, and exponents; every other page stays."""
    pages = 300
    cfg = kv_config(2, 200 * page, pages, page=page, heads=heads, group=1, dim=dim, form=form)
    tables, cache = KvTables(cfg), KvCache(cfg)
    gen = torch.Generator(device="cuda").manual_seed(5)
    cache.buffer.copy_(torch.randint(0, 256, cache.buffer.shape, generator=gen, device="cuda", dtype=torch.uint8))
    order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
    table = torch.zeros(2, 200, dtype=torch.int32, device="cuda")
    table[0] = order[:200]
    tables.load(ints([200 * page, 0]), table, order[200:].contiguous())
    want_codes, want_exps = cache.codes.clone(), cache.exps.clone()
    edit = tables.compact()
    moves = edit.moves[:int(edit.counters[6])].long()
    assert moves.shape[0] > 20
    want_codes[moves[:, 1]], want_exps[moves[:, 1]] = want_codes[moves[:, 0]], want_exps[moves[:, 0]]
    cache.copy(edit)
    assert torch.equal(cache.codes, want_codes) and torch.equal(cache.exps, want_exps)
    cache.copy(edit)
    assert torch.equal(cache.codes, want_codes) and torch.equal(cache.exps, want_exps)


def test_copies_past_four_gigabytes():
    """Pages whose bytes lie beyond 32 bits."""
    cfg = kv_config(1, 128, 5200, page=128, heads=16, group=1, dim=256)
    tables, cache = KvTables(cfg), KvCache(cfg)
    assert cache.nbytes > 5 << 30
    cache.codes[5199].random_(0, 256)
    cache.exps[5199] = torch.arange(32, device="cuda").view(16, 2).int()
    tables.load(ints([128]), ints([[5199]]), torch.arange(5199, device="cuda", dtype=torch.int32))
    edit = tables.compact()
    cache.copy(edit)
    tables.commit(edit)
    assert torch.equal(cache.codes[0], cache.codes[5199]) and torch.equal(cache.exps[0], cache.exps[5199])
    assert tables.table.tolist() == [[0]]


def test_a_plan_ends_nobody_while_pages_are_shared():
    both = Both(4, 4, 20, seed=1)
    both.window([20, 33, 0, 0])
    both.edit("fork", [0], [2], [16])
    both.window([-1, 1, -1, 2])                     # both ends refused, and counted
    assert both.node.lengths == [20, 34, 16, 2]
    both.same_tokens()
    both.edit("trim", [0, -1, -1, -1])
    both.window([0, -1, -1, 0])
    assert both.node.lengths == [0, 0, 0, 2]


def test_more_than_a_thousand_requests_end_nobody_either():
    both = Both(1500, 2, 1600, seed=2)
    both.window([17] + [1] * 500 + [0] * 999)
    both.edit("fork", [0], [1400], None)
    both.window([-1, -1] + [1] * 1498)
    assert both.node.lengths[:3] == [17, 1, 2]


def test_on_a_stream_of_its_own():
    """Work on another stream than the current one, and memory that belongs to it."""
    stream = torch.cuda.Stream()
    cfg = kv_config(8, 64, 40, heads=2, group=1, dim=64)
    tables, cache = KvTables(cfg, stream=stream), KvCache(cfg, stream=stream)
    add, src, dst, keep = ints([30] + [0] * 7), ints([0, 0]), ints([3, 5]), ints([0] + [-1] * 7)
    torch.cuda.synchronize()
    step = tables.plan(add, 30)
    tables.commit(step)
    edit = tables.fork(src, dst)
    cache.copy(edit)
    tables.commit(edit)
    tables.commit(tables.trim(keep))
    stream.synchronize()
    assert tables.lengths.tolist() == [0, 0, 0, 30, 0, 30, 0, 0] and tables.counters.tolist()[:3] == [4, 37, 1]
    assert tables.owners.tolist() == [1] + [0] * 39


def test_recorded_into_a_graph():
    """A window of samples as a graph: fork, copy, commit, end; replayed with other requests, between eager work."""
    both = Both(12, 4, 60, seed=9)
    both.window([40, 25, 0, 7] + [0] * 8)
    t, cache = both.tables, both.cache
    src, dst, tokens, keep = ints([0, 1]), ints([4, 5]), ints([40, 25]), ints([-1] * 4 + [0] * 8)
    edit, end = t.fork(src, dst, tokens), t.trim(keep)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        t.fork(src, dst, tokens, edit=edit)
        cache.copy(edit)
        t.commit(edit)
        t.trim(keep, edit=end)
        t.commit(end)
    for a, b, n in (([0, 1], [4, 5], [40, 25]), ([3, 0], [9, 10], [7, 39]), ([1, 1], [6, 11], [25, 16])):
        for x, y in ((src, a), (dst, b), (tokens, n)):
            x.copy_(ints(y))
        graph.replay()
        fork = both.node.fork(a, b, n)
        assert edit.granted.tolist() == n and edit.moves.tolist() == fork["moves"]
        both.node.commit_edit(fork)
        trim = both.node.trim([-1] * 4 + [0] * 8)
        both.node.commit_edit(trim)
        same_tables(t, both.node)
        torch.zeros(1 << 20, device="cuda").sum()
        torch.cuda.synchronize()


def test_tables_whose_numbers_are_out_of_range():
    """Page numbers that no pool has and lengths that no row has are held to the pool and the row."""
    tables, cache, _ = make(5, 3, 10)
    tables.table.copy_(ints([[-5, 1 << 30, 99]] * 5))
    tables.lengths.copy_(ints([1 << 30, -7, 48, 0, 0]))
    tables.counters.copy_(ints([-3, 1 << 20, 5, 0, 0, 0, 0, 0]))
    tables.ring.copy_(ints([1 << 29] * 10))
    for plan in (lambda: tables.fork(ints([0, 2, -9]), ints([3, 4, 1 << 30])), lambda: tables.trim(ints([3, 0, 16, -1, -1])),
                 tables.compact):
        edit = plan()
        cache.copy(edit)
        tables.commit(edit)
    torch.cuda.synchronize()
    assert all(-1 <= x < 10 for x in tables.compact().moves.flatten().tolist())


def test_c_calls_on_the_null_stream():
    """The C entry points with a null stream, as a plain C caller has them."""
    tables, cache, node = make(3, 2, 8)
    lib, c = L.lib(), ctypes.byref(tables.cfg)
    edit = KvEdit(tables.cfg, 4)
    step = tables.plan(ints([20, 0, 0]), 20)
    tables.commit(step)
    src, dst = ints([0]), ints([2])
    torch.cuda.synchronize()
    e = (edit.ptr, edit.nbytes, 4)
    assert lib.agft_pages_fork(c, tables.ptr, tables.nbytes, src.data_ptr(), dst.data_ptr(), None, 1, *e, None) == 0
    assert lib.agft_pages_copy(c, cache.ptr, cache.nbytes, *e, None) == 0
    assert lib.agft_pages_commit(c, tables.ptr, tables.nbytes, *e, None) == 0
    torch.cuda.synchronize()
    assert tables.lengths.tolist() == [20, 0, 20] and edit.moves.tolist()[0] == [1, 2]
    assert tables.table.tolist()[2] == [0, 2] and tables.owners.tolist() == [1] + [0] * 7

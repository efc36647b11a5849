"""In which order windows, edits and layers' calls may follow one another (CPU: calls
that would launch are noted by kv_stub.py instead)."""
import contextlib

import pytest
import torch

import kv_stub
from paper_2508_01744_amd import KvCache, KvTables, _lib as L, kv, kv_config

BASE = dict(requests=8, row_tokens=512, pages=200, page=16, heads=8, group=4, dim=64, form="e4m3")
ADD = torch.ones(8, dtype=torch.int32)
KEEP = torch.full((8,), -1, dtype=torch.int32)
K = torch.zeros(8, 8, 64, dtype=torch.bfloat16)
Q = torch.zeros(8, 32, 64, dtype=torch.bfloat16)


@pytest.fixture
def lib(monkeypatch):
    stub = kv_stub.install(monkeypatch)
    real = type(stub).__getattr__

    def get(self, name):
        if name.startswith("agft_pages_") and name[11:] in ("fork", "trim", "compact", "copy", "commit"):
            return lambda *args: (self.calls.append(name[5:]), L.AGFT_OK)[1]
        if name == "agft_diff_attend":
            return lambda *args: (self.calls.append("diff"), L.AGFT_OK)[1]
        return real(self, name)
    monkeypatch.setattr(kv_stub.Lib, "__getattr__", get)
    return stub


def node():
    cfg = kv_config(**BASE)
    return KvTables(cfg), KvCache(cfg)


def ints(*x):
    return torch.tensor(x, dtype=torch.int32)


def refused(lib, call, match):
    before = list(lib.calls)
    with pytest.raises(ValueError, match=match):
        call()
    assert lib.calls == before


def test_a_step_that_a_graph_plans(lib, monkeypatch):
    """Its replays plan it again, after edits too, and nobody here sees them."""
    t, cache = node()
    other = t.plan(ADD, 8)
    with monkeypatch.context() as m:
        m.setattr(kv_stub.Device, "type", "cuda")
        m.setattr(kv, "_recording", lambda: True, raising=False)
        step = t.plan(ADD, 8)
    t.commit(t.trim(KEEP))
    cache.append(step, K, K)
    cache.attend(t, step, Q)
    cache.attend_diff(t, step, Q, torch.zeros(16))
    t.commit(step)
    refused(lib, lambda: cache.append(other, K, K), "edited")


def test_a_window_behind_which_an_edit_was_planned(lib):
    """A fork's plan writes rows, where the window's tokens had put their pages."""
    t, cache = node()
    step = t.plan(ADD, 8)
    edit = t.fork(ints(0), ints(5))
    refused(lib, lambda: t.commit(step), "planned since")
    refused(lib, lambda: cache.attend(t, step, Q), "planned since")
    refused(lib, lambda: cache.attend_diff(t, step, Q, torch.zeros(16)), "planned since")
    cache.copy(edit)
    t.commit(edit)
    refused(lib, lambda: t.commit(step), "edited")
    for other in (lambda: t.trim(KEEP), t.compact):
        t.plan(ADD, 8, step=step)
        edit = other()
        refused(lib, lambda: t.commit(step), "planned since")
        t.plan(ADD, 8, step=step)                       # (planned again, it is the latest)
        cache.append(step, K, K)
        t.commit(step)
        refused(lib, lambda: t.commit(edit), "changed")


def test_an_edit_behind_which_something_was_planned(lib):
    """Ends and trims write the ring, and forks and windows rows: the latest plan's are there."""
    t, cache = node()
    plans = (lambda: t.plan(-ADD, 8), lambda: t.trim(KEEP), t.compact, lambda: t.fork(ints(0), ints(1)))
    for first in plans[1:]:
        for second in plans:
            edit, last = first(), second()
            refused(lib, lambda: t.commit(edit), "planned since")
            refused(lib, lambda: cache.copy(edit), "has been")
            t.commit(last)


def test_a_window_behind_which_another_was_planned(lib):
    t, cache = node()
    step = t.plan(ADD, 8)
    last = t.plan(-ADD, 8)
    refused(lib, lambda: t.commit(step), "planned since")
    refused(lib, lambda: cache.append(step, K, K), "planned since")
    cache.attend(t, step, Q)
    t.commit(last)
    step = t.plan(ADD, 8)
    t.commit(step)
    last = t.plan(ADD, 8)                               # its layers may follow: the tokens are the tables'
    cache.append(step, K, K)
    cache.attend(t, step, Q)
    cache.append(last, K, K)
    t.commit(last)
    refused(lib, lambda: t.commit(step), "planned since")


def test_steps_of_other_tables_and_of_tables_that_began_anew(lib):
    t, cache = node()
    other = KvTables(t.cfg)
    step = t.plan(ADD, 8)
    refused(lib, lambda: cache.attend(other, step, Q), "other tables")
    refused(lib, lambda: cache.attend_diff(other, step, Q, torch.zeros(16)), "other tables")
    refused(lib, lambda: other.commit(step), "other tables")
    t._settled = contextlib.nullcontext
    for anew in (t.reset, lambda: t.load(torch.zeros(8, dtype=torch.int32), torch.zeros(8, 32, dtype=torch.int32), ints(1))):
        t.plan(ADD, 8, step=step)
        anew()
        for call in (lambda: cache.append(step, K, K), lambda: cache.attend(t, step, Q), lambda: t.commit(step)):
            refused(lib, call, "reset")
        edit = t.trim(KEEP)
        anew()
        refused(lib, lambda: t.commit(edit), "changed")
    t.plan(ADD, 8, step=step)
    cache.append(step, K, K)
    cache.attend(t, step, Q)
    t.commit(step)


def test_graphs_whose_plans_are_recorded(lib, monkeypatch):
    """Two graphs, each with a plan: recording runs nothing, and eager calls follow either's replays."""
    t, cache = node()
    open_ = t.plan(ADD, 8)
    with monkeypatch.context() as m:
        m.setattr(kv_stub.Device, "type", "cuda")
        m.setattr(kv, "_recording", lambda: True)
        steps = [t.plan(ADD, 8) for _ in range(2)]
    t.commit(open_)
    for step in (*steps, *steps):
        cache.append(step, K, K)
        cache.attend(t, step, Q)
        t.commit(step)


def test_a_layers_copies_come_before_its_tokens_of_later_windows(lib):
    """The copy would write over a token in a fork's last page, or copy a page that was filled anew."""
    t, cache = node()
    late = KvCache(t.cfg)
    edit = t.fork(ints(0, 1), ints(5, 6))
    t.commit(edit)
    step = t.plan(ADD, 8)
    cache.copy(edit)                                    # (a plan writes to no layer)
    for layer in (cache, late):
        layer.append(step, K, K)
    refused(lib, lambda: late.copy(edit), "already")
    refused(lib, lambda: cache.copy(edit), "already")
    KvCache(t.cfg).copy(edit)
    other = KvTables(t.cfg)                             # (other tables' windows say nothing of these)
    for _ in range(3):
        other.commit(other.plan(ADD, 8))
    step = other.plan(ADD, 8)
    free = KvCache(t.cfg)
    free.append(step, K, K)
    free.copy(edit)


def test_a_layers_tokens_of_earlier_windows_come_before_its_copies(lib):
    """A fork's last page would lack them, and a moved page too."""
    t, cache = node()
    step = t.plan(ADD, 8)
    t.commit(step)
    for plan in (t.compact, lambda: t.fork(ints(0), ints(1))):
        edit = plan()
        late = KvCache(t.cfg)
        late.append(step, K, K)
        late.copy(edit)
        refused(lib, lambda: late.append(step, K, K), "copied in this layer")
    t.commit(edit)
    step = t.plan(ADD, 8)
    late.append(step, K, K)
    t.commit(step)

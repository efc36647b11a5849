"""In which order windows, edits and layers' calls may follow one another (CPU: calls
that would launch are noted by kv_stub.py instead)."""
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

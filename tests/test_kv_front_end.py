"""What the cache's front end refuses before anything is enqueued (CPU: calls
that would launch are noted by kv_stub.py instead)."""
import contextlib
import weakref
from types import SimpleNamespace

import pytest
import torch

import kv_stub
from paper_2508_01744_amd import KvCache, KvStep, KvTables, kv, kv_config


@pytest.fixture
def lib(monkeypatch):
    return kv_stub.install(monkeypatch)


BASE = dict(requests=64, row_tokens=512, pages=200, page=16, heads=8, group=4, dim=64, form="e4m3")


def tensors(cfg, n=32, dtype=torch.bfloat16):
    k = torch.zeros(n, cfg.heads, cfg.dim, dtype=dtype)
    return k, torch.zeros(n, cfg.heads * cfg.group, cfg.dim, dtype=dtype)


def refused(lib, call, match):
    before = list(lib.calls)
    with pytest.raises(ValueError, match=match):
        call()
    assert lib.calls == before


@pytest.mark.parametrize("other", [dict(heads=16), dict(heads=4), dict(group=8), dict(group=2), dict(page=32),
                                   dict(requests=65), dict(requests=63), dict(pages=201), dict(row_tokens=528),
                                   dict(row_tokens=256)])
def test_objects_of_other_configurations(lib, other):
    """A step's and the tables' parts lie where their configuration puts them."""
    cfg, cfg2 = kv_config(**BASE), kv_config(**{**BASE, **other})
    tables, tables2, cache, cache2 = KvTables(cfg), KvTables(cfg2), KvCache(cfg), KvCache(cfg2)
    add, add2 = (torch.ones(c.requests, dtype=torch.int32) for c in (cfg, cfg2))
    step = tables.plan(add, 32)
    tables2.plan(add2, 32)
    k2, q2 = tensors(cfg2)
    k, q = tensors(cfg)
    refused(lib, lambda: cache2.append(step, k2, k2), "configuration")
    refused(lib, lambda: cache2.attend(tables2, step, q2), "configuration")
    refused(lib, lambda: cache2.attend(tables, step, q2), "configuration")
    refused(lib, lambda: cache.attend(tables2, step, q), "configuration")
    refused(lib, lambda: tables2.plan(add2, 32, step=step), "configuration")
    refused(lib, lambda: tables2.commit(step), "configuration")
    del lib.calls[:]
    cache.append(step, k, k)
    cache.attend(tables, step, q)
    tables.commit(step)
    assert lib.calls == ["append", "attend", "commit"]


def test_layers_may_differ_in_what_the_tables_do_not_hold(lib):
    """One set of tables and one step for layers of other forms and smaller heads."""
    cfg = kv_config(**{**BASE, "dim": 256})
    tables = KvTables(cfg)
    step = tables.plan(torch.ones(64, dtype=torch.int32), 32)
    for kw in (dict(dim=256, form="int8"), dict(dim=128), dict(dim=64, form="int8")):
        other = kv_config(**{**BASE, **kw})
        k, q = tensors(other)
        cache = KvCache(other)
        cache.append(step, k, k)
        cache.attend(tables, step, q)


def test_a_configuration_that_is_changed_later(lib):
    """Objects keep the configuration that they were made with."""
    cfg = kv_config(**BASE)
    tables, cache = KvTables(cfg), KvCache(cfg)
    cfg.heads, cfg.requests = 16, 9
    assert tables.cfg.heads == cache.cfg.heads == 8
    step = tables.plan(torch.ones(64, dtype=torch.int32), 32)
    assert isinstance(step, KvStep) and step.cfg.requests == 64
    k, q = tensors(cache.cfg)
    cache.append(step, k, k)
    cache.attend(tables, step, q)


def test_the_workspace_fits_the_largest_layer(lib):
    """Layers of growing heads on one step: each gets a workspace as large as it needs."""
    cfg = kv_config(**BASE)
    tables = KvTables(cfg)
    step = tables.plan(torch.ones(64, dtype=torch.int32), 32)
    seen = []
    for dim in (64, 256, 128, 256):
        cache = KvCache(kv_config(**{**BASE, "dim": dim}))
        cache.attend(tables, step, tensors(cache.cfg)[1])
        work, nbytes = lib.args[-1][-3:-1]
        assert nbytes >= lib.real.agft_kv_attend_bytes(cache._cfg, 32)
        seen.append(work)
    assert seen[1] == seen[2] == seen[3]


def test_a_step_that_was_never_planned(lib):
    """Its memory holds anything, and the kernels take indices from it."""
    cfg = kv_config(**BASE)
    tables, cache = KvTables(cfg), KvCache(cfg)
    k, q = tensors(cfg)
    step = KvStep(cfg, 32)
    refused(lib, lambda: cache.append(step, k, k), "planned")
    refused(lib, lambda: cache.attend(tables, step, q), "planned")
    refused(lib, lambda: tables.commit(step), "planned")
    with pytest.raises(ValueError):
        tables.plan(torch.ones(63, dtype=torch.int32), 32, step=step)
    refused(lib, lambda: cache.append(step, k, k), "planned")
    tables.plan(torch.ones(64, dtype=torch.int32), 32, step=step)
    cache.append(step, k, k)
    cache.attend(tables, step, q)
    tables.commit(step)


def test_launches_go_to_the_objects_device(lib, monkeypatch):
    """A launch takes the calling thread's current device: with another one current
    the kernels would run there, on memory of this one."""
    cfg = kv_config(**BASE)
    tables, cache = KvTables(cfg), KvCache(cfg)
    add = torch.ones(64, dtype=torch.int32)
    step = tables.plan(add, 32)
    k, q = tensors(cfg)
    slots = torch.zeros(5, dtype=torch.int64)
    monkeypatch.setattr(kv, "_current_device", lambda: 3)
    for call in (lambda: tables.plan(add, 32, step=step), lambda: cache.append(step, k, k),
                 lambda: cache.attend(tables, step, q), lambda: tables.commit(step), lambda: cache.export(slots),
                 tables.reset, lambda: KvTables(cfg)):
        refused(lib, call, "current device")


def test_objects_and_streams_of_other_devices(lib):
    cfg = kv_config(**BASE)
    tables, cache = KvTables(cfg), KvCache(cfg)
    step = tables.plan(torch.ones(64, dtype=torch.int32), 32)
    k, q = tensors(cfg)
    stream = SimpleNamespace(device=torch.device("cuda", 3), cuda_stream=0)
    refused(lib, lambda: cache.set_stream(stream), "cuda:3")
    refused(lib, lambda: KvCache(cfg, stream=stream), "cuda:3")
    tables.device = torch.device("cuda", 3)
    refused(lib, lambda: cache.attend(tables, step, q), "cuda:3")
    step.device = torch.device("cuda", 3)
    refused(lib, lambda: cache.append(step, k, k), "cuda:3")


def test_older_workspaces_stay(lib):
    """A recorded graph may hold the one that a larger layer's replaced."""
    cfg = kv_config(**BASE)
    tables = KvTables(cfg)
    step = tables.plan(torch.ones(64, dtype=torch.int32), 32)
    small = weakref.ref(step.work(KvCache(cfg)))
    big = step.work(KvCache(kv_config(**{**BASE, "dim": 256})))
    assert small() is not None and step.work() is big


@pytest.mark.parametrize("bad", [-127, -200, 127, 128, 2 ** 31 - 1, -2 ** 31])
def test_exponents_that_are_none(lib, monkeypatch, bad):
    """A scale of 2^e, and of 2^-e, has to be a number of fp32."""
    monkeypatch.setattr(kv._OnStream, "_settled", lambda self: contextlib.nullcontext())
    cfg = kv_config(**{**BASE, "pages": 3})
    cache = KvCache(cfg)
    codes = torch.randint(0, 100, (3, 8, 2, 16, 64), dtype=torch.uint8)
    exps = torch.randint(-126, 127, (3, 8, 2), dtype=torch.int32)
    exps[0, 0, 0], exps[0, 0, 1] = -126, 126
    cache.load(codes, exps)
    held = cache.buffer.clone()
    exps[2, 5, 1] = bad
    refused(lib, lambda: cache.load(codes + 1, exps), "exponents")
    assert torch.equal(cache.buffer, held)


def test_no_gradient_is_lost_in_silence(lib):
    """There is no backward pass: inputs that ask for one are refused."""
    cfg = kv_config(**BASE)
    tables, cache = KvTables(cfg), KvCache(cfg)
    step = tables.plan(torch.ones(64, dtype=torch.int32), 32)
    k, q = tensors(cfg)
    for t in (k, q):
        t.requires_grad_()
    refused(lib, lambda: cache.append(step, k, k.detach()), "gradient")
    refused(lib, lambda: cache.append(step, k.detach(), k), "gradient")
    refused(lib, lambda: cache.attend(tables, step, q), "gradient")
    refused(lib, lambda: cache.attend(tables, step, q * 1), "gradient")
    refused(lib, lambda: cache.attend(tables, step, q.detach(), out=q), "gradient")
    with torch.no_grad():
        cache.append(step, k, k)
        cache.attend(tables, step, q)
    with torch.inference_mode():
        cache.attend(tables, step, q)
    cache.append(step, k.detach(), k.detach())
    cache.attend(tables, step, q.detach())

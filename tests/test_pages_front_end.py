"""What the calls that edit a cache's tables refuse before anything is enqueued,
their C ABI and launches (CPU: calls that would launch are noted instead)."""
import ctypes
import os
import re

import pytest
import torch

import kv_stub
from paper_2508_01744_amd import KvCache, KvEdit, KvTables, kv_config, lib as load
from paper_2508_01744_amd import _lib as L

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BASE = dict(requests=8, row_tokens=512, pages=200, page=16, heads=8, group=4, dim=64, form="e4m3")
EDITS = ("fork", "trim", "compact", "copy", "commit")


@pytest.fixture
def lib(monkeypatch):
    stub = kv_stub.install(monkeypatch)
    real = type(stub).__getattr__

    def get(self, name):
        if name.startswith("agft_pages_") and name[11:] in EDITS:
            return lambda *args: (self.calls.append("pages " + name[11:]), L.AGFT_OK)[1]
        return real(self, name)
    monkeypatch.setattr(kv_stub.Lib, "__getattr__", get)
    return stub


def ints(*x):
    return torch.tensor(x, dtype=torch.int32)


def refused(lib, call, match):
    before = list(lib.calls)
    with pytest.raises(ValueError, match=match):
        call()
    assert lib.calls == before


def test_every_declared_symbol_is_exported():
    text = open(os.path.join(ROOT, "include", "agft_pages.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = set(re.findall(r"^\s*(?:const\s+)?[a-z_0-9]+\s*\**\s*(agft_pages_[a-z_0-9]+)\s*\(", text, flags=re.M))
    assert names == set(L.PAGES_EXPORTED) and len(names) == 8
    for n in names:
        assert hasattr(load(), n), n


def test_arguments(lib):
    t = KvTables(kv_config(**BASE))
    a, b = ints(0, 1), ints(2, 3)
    refused(lib, lambda: t.fork(a, ints(2)), "dst")
    refused(lib, lambda: t.fork(a.long(), b), "src")
    refused(lib, lambda: t.fork(a[:0], b[:0]), "1 to 65536")
    refused(lib, lambda: t.fork(a.view(1, 2), b), "1 to 65536")
    refused(lib, lambda: t.fork(ints(0, 1, 2, 3)[::2], b), "contiguous")
    refused(lib, lambda: t.fork(a, b, ints(1)), "tokens")
    refused(lib, lambda: t.fork(a, b, a.float()), "tokens")
    refused(lib, lambda: t.trim(ints(1, 2)), "keep")
    refused(lib, lambda: t.fork(a, b, edit=KvEdit(t.cfg, 3)), "3 moves")
    refused(lib, lambda: t.compact(edit=KvEdit(t.cfg, 3)), "3 moves")
    for n in (0, -1, (1 << 27) + 1):
        refused(lib, lambda: KvEdit(t.cfg, n), "max_moves")
    other = KvTables(kv_config(**{**BASE, "pages": 201}))
    others = other.fork(a, b)
    refused(lib, lambda: t.fork(a, b, edit=others), "configuration")
    refused(lib, lambda: t.commit(others), "configuration")
    refused(lib, lambda: KvCache(t.cfg).copy(others), "configuration")
    refused(lib, lambda: KvCache(t.cfg).copy(KvEdit(t.cfg, 2)), "not been planned")
    refused(lib, lambda: t.commit(KvEdit(t.cfg, 2)), "not been planned")


def test_layers_may_differ(lib):
    t = KvTables(kv_config(**BASE))
    edit = t.compact()
    assert edit.max_moves == 100 and edit.moves.shape == (100, 2) and edit.lengths.shape == (8,)
    for kw in (dict(dim=256, form="int8"), dict(dim=128)):
        KvCache(kv_config(**{**BASE, **kw})).copy(edit)
    t.commit(edit)
    assert lib.calls[-4:] == ["pages compact", "pages copy", "pages copy", "pages commit"]
    assert KvTables(kv_config(**{**BASE, "pages": 1})).compact().max_moves == 1


def test_an_edit_is_for_the_tables_that_it_was_planned_from(lib):
    t = KvTables(kv_config(**BASE))
    first, second = t.trim(ints(*[-1] * 8)), t.compact()
    t.commit(second)
    refused(lib, lambda: t.commit(first), "changed")
    refused(lib, lambda: t.commit(second), "changed")               # (once is enough)
    t.commit(t.trim(ints(*[-1] * 8), edit=first))
    again = t.compact(edit=second)
    t.commit(t.plan(ints(*[1] * 8), 8))
    refused(lib, lambda: t.commit(again), "changed")
    again = t.compact(edit=second)
    t.reset()
    refused(lib, lambda: t.commit(again), "changed")
    refused(lib, lambda: KvCache(t.cfg).copy(again), "changed")     # (its pages may be others' by now)
    t.compact(edit=second)
    cache = KvCache(t.cfg)
    cache.copy(second)
    t.commit(second)
    cache.copy(second)                                              # (another layer)
    t.commit(t.plan(ints(*[1] * 8), 8))
    refused(lib, lambda: cache.copy(second), "changed")
    t.compact(edit=second)
    apart = KvTables(t.cfg)
    refused(lib, lambda: apart.commit(second), "not theirs")


def test_a_window_is_for_the_tables_that_it_was_planned_from(lib):
    """After an edit a step's slots and lengths are those of other pages."""
    cfg = kv_config(**BASE)
    t, cache = KvTables(cfg), KvCache(cfg)
    k, q = torch.zeros(8, 8, 64, dtype=torch.bfloat16), torch.zeros(8, 32, 64, dtype=torch.bfloat16)
    add = ints(*[1] * 8)
    step = t.plan(add, 8)
    edit = t.compact()
    cache.append(step, k, k)
    t.commit(edit)
    for call in (lambda: cache.append(step, k, k), lambda: cache.attend(t, step, q), lambda: t.commit(step)):
        refused(lib, call, "edited")
    t.plan(add, 8, step=step)
    cache.append(step, k, k)
    cache.attend(t, step, q)
    t.commit(step)
    t.commit(step)


def test_loading_shared_tables(lib):
    cfg = kv_config(**{**BASE, "requests": 3, "row_tokens": 64})
    t = KvTables(cfg)
    table = ints(5, 6, 7, 9, 5, 6, 8, 0, 5, 9, 9, 9).view(3, 4)
    import contextlib
    t._settled = contextlib.nullcontext
    t.load(ints(48, 33, 16), table, ints(1, 2, 3), shared=True)
    want = torch.zeros(200, dtype=torch.int32)
    want[5], want[6] = 2, 1
    assert torch.equal(t.owners, want) and t.counters.tolist() == [0, 3, 3, 0, 0, 0, 0, 0]
    t.load(ints(48, 33, 16), table, ints(1, 2, 3))
    assert not t.owners.any() and t.counters.tolist()[2] == 0


P, ODD, BIG = ctypes.c_void_p(0x100000), ctypes.c_void_p(0x100002), 1 << 40


def test_c_calls_reject_before_launch():
    lib, c, E = load(), ctypes.byref(kv_config(**BASE)), L.AGFT_E_INVAL
    bytes_ = lib.agft_pages_edit_bytes
    assert bytes_(c, 1) > 0 and bytes_(c, 1 << 27) > 1 << 30
    assert [bytes_(c, n) for n in (0, -1, (1 << 27) + 1)] == [0, 0, 0] and bytes_(None, 1) == 0
    v, n = L.agft_pages_view(), bytes_(c, 9)
    assert lib.agft_pages_edit_at(c, 9, P, n, ctypes.byref(v)) == 0 and v.moves + 72 <= P.value + n
    for args in ((9, P, n - 1, ctypes.byref(v)), (9, P, n, None), (9, None, n, ctypes.byref(v)), (0, P, n, ctypes.byref(v)),
                 (9, ctypes.c_void_p(0x100010), n, ctypes.byref(v))):
        assert lib.agft_pages_edit_at(c, *args) == E
    o = ctypes.c_void_p()
    assert lib.agft_pages_owners_at(c, P, BIG, None) == E and lib.agft_pages_owners_at(c, P, 64, ctypes.byref(o)) == E
    e = (P, BIG, 100)
    for src, dst, tok, m in ((None, P, None, 1), (P, None, None, 1), (ODD, P, None, 1), (P, ODD, None, 1), (P, P, ODD, 1),
                             (P, P, None, 0), (P, P, None, -1), (P, P, None, 101)):
        assert lib.agft_pages_fork(c, P, BIG, src, dst, tok, m, *e, None) == E
    assert lib.agft_pages_fork(c, P, BIG, P, P, None, 65537, P, BIG, 70000, None) == E
    assert lib.agft_pages_trim(c, P, BIG, None, *e, None) == E and lib.agft_pages_trim(c, P, BIG, ODD, *e, None) == E
    assert lib.agft_pages_compact(c, P, BIG, P, BIG, 99, None) == E
    for f, args in ((lib.agft_pages_trim, (P,)), (lib.agft_pages_compact, ()), (lib.agft_pages_commit, ())):
        assert f(c, None, BIG, *args, *e, None) == E and f(c, P, 100, *args, *e, None) == E
        assert f(c, P, BIG, *args, None, BIG, 100, None) == E and f(c, P, BIG, *args, P, 100, 100, None) == E
        assert f(c, P, BIG, *args, P, BIG, 0, None) == E
        u = ctypes.byref(kv_config(**{**BASE, "dim": 96}))
        assert f(u, P, BIG, *args, *e, None) == L.AGFT_E_UNSUPPORTED
    assert lib.agft_pages_copy(c, None, BIG, *e, None) == E and lib.agft_pages_copy(c, P, 100, *e, None) == E
    assert lib.agft_pages_copy(c, P, BIG, P, 100, 100, None) == E


def test_no_kernel_spills(tmp_path):
    import subprocess
    from paper_2508_01744_amd import _build
    from test_kv_build import HIPCC
    if not os.path.exists(HIPCC):
        pytest.skip("hipcc not found")
    flags = [f for f in _build.HIPCC_FLAGS if f != "-shared"]
    out = subprocess.run([HIPCC, *flags, "--cuda-device-only", "-c", "-I", _build.INCLUDE,
                          os.path.join(_build.CSRC, "agft_pages.hip"), "-o", str(tmp_path / "pages.o"),
                          "-Rpass-analysis=kernel-resource-usage"], capture_output=True, text=True, check=True).stderr
    kernels = re.findall(r"Function Name: (\S+)(.*?)(?=Function Name:|\Z)", out, re.S)
    assert len(kernels) >= 12
    for name, body in kernels:
        scratch, vector = (int(re.search(p + r": (\d+)", body).group(1)) for p in (r"ScratchSize \[bytes/lane\]", "VGPRs Spill"))
        assert scratch == 0 and vector == 0, name

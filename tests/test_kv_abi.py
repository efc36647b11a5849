"""The cache's C ABI: exported symbols, buffer sizes, and arguments rejected
before anything is enqueued (CPU only: no call here launches work)."""
import ctypes
import os
import re

import pytest

import paper_2508_01744_amd._lib as L
from kv_reference import exponent, held
from paper_2508_01744_amd import kv_config

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = ctypes.c_void_p(0x100000)
ODD = ctypes.c_void_p(0x100010)
BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    return L.lib()


def cfg(**kw):
    args = dict(requests=3, row_tokens=1000, pages=40, page=16, heads=2, group=4, dim=128, form="e4m3")
    raw = {k: kw.pop(k) for k in ("row_pages", "form_raw") if k in kw}
    args.update(kw)
    c = kv_config(**args)
    if "row_pages" in raw:
        c.row_pages = raw["row_pages"]
    if "form_raw" in raw:
        c.form = raw["form_raw"]
    return c


def test_every_declared_symbol_is_exported(lib):
    text = open(os.path.join(ROOT, "include", "agft_kv.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = set(re.findall(r"^\s*(?:const\s+)?[a-z_0-9]+\s*\**\s*(agft_kv_[a-z_0-9]+)\s*\(", text, flags=re.M))
    assert names == set(L.KV_EXPORTED) and len(names) == 12
    for n in names:
        assert hasattr(lib, n), n


def test_buffer_sizes(lib):
    c = cfg()
    b = ctypes.byref(c)
    assert c.row_pages == 63
    assert lib.agft_kv_tables_bytes(b) >= 4 * (8 + 3 + 3 * 63 + 40) and lib.agft_kv_tables_bytes(b) % 256 == 0
    codes = 40 * 2 * 2 * 16 * 128
    assert codes + 40 * 2 * 2 * 4 <= lib.agft_kv_cache_bytes(b) < codes + 40 * 2 * 2 * 4 + 512
    assert lib.agft_kv_step_bytes(b, 100) >= 100 * 8 + 4 * (8 + 4 + 3 + 3)
    assert lib.agft_kv_attend_bytes(b, 100) > 0
    big = cfg(pages=1 << 28, heads=256, dim=256, page=128)
    assert lib.agft_kv_cache_bytes(ctypes.byref(big)) > (1 << 28) * 256 * 2 * 128 * 256   # (64 bits hold it)
    for n in (0, -1, (1 << 30) + 1):
        assert lib.agft_kv_step_bytes(b, n) == 0 and lib.agft_kv_attend_bytes(b, n) == 0
    for bad in (dict(requests=0), dict(requests=65537), dict(row_pages=0), dict(row_pages=1 << 26), dict(pages=0),
                dict(pages=(1 << 28) + 1), dict(page=8), dict(page=24), dict(page=256), dict(heads=0), dict(heads=257),
                dict(group=0), dict(group=129), dict(dim=0), dict(dim=96), dict(form_raw=2), dict(form_raw=-1)):
        c = ctypes.byref(cfg(**bad))
        assert lib.agft_kv_tables_bytes(c) == lib.agft_kv_cache_bytes(c) == lib.agft_kv_step_bytes(c, 5) == 0, bad
    assert lib.agft_kv_cache_bytes(None) == 0


def test_views(lib):
    c = cfg()
    b = ctypes.byref(c)
    n = lib.agft_kv_tables_bytes(b)
    v = L.agft_kv_tables_view()
    assert lib.agft_kv_tables_at(b, P, n, ctypes.byref(v)) == 0
    assert v.counters == P.value and v.ring + 40 * 4 <= P.value + n
    assert lib.agft_kv_tables_at(b, P, n - 1, ctypes.byref(v)) == L.AGFT_E_INVAL
    assert lib.agft_kv_tables_at(b, ODD, n, ctypes.byref(v)) == L.AGFT_E_INVAL
    assert lib.agft_kv_tables_at(b, None, n, ctypes.byref(v)) == L.AGFT_E_INVAL
    assert lib.agft_kv_tables_at(b, P, n, None) == L.AGFT_E_INVAL
    assert lib.agft_kv_tables_at(None, P, n, ctypes.byref(v)) == L.AGFT_E_INVAL
    m = lib.agft_kv_step_bytes(b, 9)
    s = L.agft_kv_step_view()
    assert lib.agft_kv_step_at(b, 9, P, m, ctypes.byref(s)) == 0 and s.slots + 9 * 8 <= P.value + m
    assert lib.agft_kv_step_at(b, 10 ** 6, P, m, ctypes.byref(s)) == L.AGFT_E_INVAL
    assert lib.agft_kv_step_at(b, 0, P, m, ctypes.byref(s)) == L.AGFT_E_INVAL
    u = ctypes.byref(cfg(dim=96))
    assert lib.agft_kv_tables_at(u, P, BIG, ctypes.byref(v)) == L.AGFT_E_UNSUPPORTED
    assert lib.agft_kv_step_at(u, 9, P, BIG, ctypes.byref(s)) == L.AGFT_E_UNSUPPORTED


def dense(data=0x200000, token=256, head=128, type_=L.AGFT_KV_BF16):
    return ctypes.byref(L.agft_kv_dense(data, token, head, type_))


def test_calls_reject_before_launch(lib):
    c = ctypes.byref(cfg())
    E = L.AGFT_E_INVAL
    assert lib.agft_kv_reset(c, None, BIG, None) == E and lib.agft_kv_reset(c, P, 100, None) == E
    assert lib.agft_kv_plan(c, P, BIG, None, P, BIG, 9, None) == E
    assert lib.agft_kv_plan(c, P, BIG, ctypes.c_void_p(0x100002), P, BIG, 9, None) == E
    assert lib.agft_kv_plan(c, None, BIG, P, P, BIG, 9, None) == E
    assert lib.agft_kv_plan(c, P, BIG, P, P, 64, 9, None) == E
    assert lib.agft_kv_plan(c, P, BIG, P, P, BIG, 0, None) == E
    assert lib.agft_kv_plan(ctypes.byref(cfg(dim=48)), P, BIG, P, P, BIG, 9, None) == L.AGFT_E_UNSUPPORTED
    assert lib.agft_kv_commit(c, P, BIG, None, BIG, 9, None) == E
    assert lib.agft_kv_commit(c, P, 1, P, BIG, 9, None) == E
    good = dense()
    bads = (dense(0), dense(0x200008), dense(token=257), dense(head=4), dense(type_=3), dense(token=-256), None)
    for bad in bads:
        assert lib.agft_kv_append(c, P, BIG, P, BIG, 9, bad, good, None) == E
        assert lib.agft_kv_append(c, P, BIG, P, BIG, 9, good, bad, None) == E
        assert lib.agft_kv_attend(c, P, BIG, P, BIG, P, BIG, 9, 9, bad, good, None, 1.0, P, BIG, None) == E
        assert lib.agft_kv_attend(c, P, BIG, P, BIG, P, BIG, 9, 9, good, bad, None, 1.0, P, BIG, None) == E
        assert lib.agft_kv_export(c, P, BIG, P, 5, bad, good, None) == E
        assert lib.agft_kv_export(c, P, BIG, P, 5, good, bad, None) == E
    half = dense(type_=L.AGFT_KV_FP16)
    assert lib.agft_kv_append(c, P, BIG, P, BIG, 9, good, half, None) == E
    assert lib.agft_kv_append(c, P, 100, P, BIG, 9, good, good, None) == E
    assert lib.agft_kv_append(c, None, BIG, P, BIG, 9, good, good, None) == E

    def attend(q=good, out=good, lse=None, scale=1.0, n=9, new=9, cache=P, work=P, wbytes=BIG, tables=P, step=P):
        return lib.agft_kv_attend(c, cache, BIG, tables, BIG, step, BIG, n, new, q, out, lse, scale, work, wbytes, None)

    wide = dense(type_=L.AGFT_KV_FP32)
    for kw in (dict(q=good, out=half), dict(q=wide, out=wide), dict(lse=ctypes.c_void_p(0x100001)),
               dict(scale=float("nan")), dict(scale=float("inf")), dict(new=0), dict(new=10), dict(n=0), dict(cache=None),
               dict(work=None), dict(work=ODD), dict(wbytes=0), dict(tables=ODD), dict(step=None)):
        assert attend(**kw) == E, kw
    assert lib.agft_kv_export(c, P, BIG, None, 5, good, good, None) == E
    assert lib.agft_kv_export(c, P, BIG, P, -1, good, good, None) == E
    assert lib.agft_kv_export(c, P, BIG, ctypes.c_void_p(0x100004), 5, good, good, None) == E
    assert lib.agft_kv_export(c, P, 100, P, 5, good, good, None) == E
    assert lib.agft_kv_export(c, P, BIG, None, 0, None, None, None) == L.AGFT_OK    # nothing to do


def test_reference_codes():
    """The reference's own rounding at known numbers of e4m3 and of integers."""
    assert held(448.0, "e4m3") == 448 and held(17.0, "e4m3") == 16 and held(19.0, "e4m3") == 20
    assert held(2.0 ** -9, "e4m3") == 2.0 ** -9 and held(2.0 ** -10, "e4m3") == 0 and held(1.0625, "e4m3") == 1.0
    assert held(2.5, "int8") == 2 and held(-3.5, "int8") == -4 and held(float("inf"), "int8") == 127
    assert exponent(448.0, "e4m3") == 0 and exponent(448.1, "e4m3") == 1 and exponent(224.0, "e4m3") == -1
    assert exponent(127.0, "int8") == 0 and exponent(0.0, "int8") == -64

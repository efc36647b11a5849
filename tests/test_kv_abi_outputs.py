"""Outputs whose rows would lie on one another are refused (CPU only: no call
here launches work)."""
import ctypes

import pytest

import paper_2508_01744_amd._lib as L
from paper_2508_01744_amd import kv_config

P = ctypes.c_void_p(0x100000)
BIG = 1 << 40


def dense(token=256, head=128):
    return ctypes.byref(L.agft_kv_dense(0x200000, token, head, L.AGFT_KV_BF16))


@pytest.mark.parametrize("bad", [dict(token=0), dict(head=0), dict(token=0, head=0)])
def test_outputs_on_one_another(bad):
    lib, c = L.lib(), ctypes.byref(kv_config(3, 1000, 40, heads=2, group=4))
    good, bad = dense(), dense(**bad)
    assert lib.agft_kv_attend(c, P, BIG, P, BIG, P, BIG, 9, 9, good, bad, None, 1.0, P, BIG, None) == L.AGFT_E_INVAL
    assert lib.agft_kv_export(c, P, BIG, P, 5, bad, good, None) == L.AGFT_E_INVAL
    assert lib.agft_kv_export(c, P, BIG, P, 5, good, bad, None) == L.AGFT_E_INVAL

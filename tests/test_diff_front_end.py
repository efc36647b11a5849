"""What differential attention refuses before anything is enqueued, its C ABI, its
kernels' registers (CPU: calls that would launch are noted instead), and its bound
on planted mistakes (in the reference)."""
import ctypes
import os
import re
import subprocess

import pytest
import torch

import kv_stub
from diff_reference import lambdas, reference, weights
from kv_flat import Window
from paper_2508_01744_amd import KvCache, KvTables, _build, kv_config, lib as load
from paper_2508_01744_amd import _lib as L
from test_kv_build import HIPCC

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BASE = dict(requests=8, row_tokens=512, pages=200, page=16, heads=8, group=4, dim=64, form="e4m3")


@pytest.fixture
def lib(monkeypatch):
    stub = kv_stub.install(monkeypatch)
    real = type(stub).__getattr__

    def get(self, name):
        if name == "agft_diff_attend":
            return lambda *args: (self.calls.append("diff"), self.args.append(args), L.AGFT_OK)[2]
        return real(self, name)
    monkeypatch.setattr(kv_stub.Lib, "__getattr__", get)
    return stub


def node(**kw):
    cfg = kv_config(**{**BASE, **kw})
    tables = KvTables(cfg)
    step = tables.plan(torch.ones(8, dtype=torch.int32), 8)
    return tables, KvCache(cfg), step, torch.zeros(8, cfg.heads * cfg.group, cfg.dim, dtype=torch.bfloat16)


def refused(lib, call, match):
    before = list(lib.calls)
    with pytest.raises(ValueError, match=match):
        call()
    assert lib.calls == before


def test_every_declared_symbol_is_exported():
    text = open(os.path.join(ROOT, "include", "agft_diff.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = set(re.findall(r"^\s*(?:const\s+)?[a-z_0-9]+\s*\**\s*(agft_diff_[a-z_0-9]+)\s*\(", text, flags=re.M))
    assert names == set(L.DIFF_EXPORTED) and len(names) == 2
    for n in names:
        assert hasattr(load(), n), n


def test_arguments(lib):
    t, cache, step, q = node()
    lam, weight = torch.zeros(16), torch.zeros(128)
    call = lambda **kw: cache.attend_diff(t, step, **{**dict(q=q, lam=lam), **kw})       # noqa: E731
    for bad in (lam[:15], lam.double(), lam.view(1, 16), torch.zeros(7, 16), torch.zeros(8, 15), torch.zeros(8, 1, 16),
                torch.tensor(0.5)):
        refused(lib, lambda: call(lam=bad), "lam must be")
    for bad in (weight[:127], weight.bfloat16(), torch.zeros(256)[::2], torch.zeros(129)[1:], torch.zeros(1, 128)):
        refused(lib, lambda: call(weight=bad), "weight must be")
    refused(lib, lambda: call(lam=lam.clone().requires_grad_()), "gradient")
    refused(lib, lambda: call(weight=weight.clone().requires_grad_()), "gradient")
    refused(lib, lambda: call(q=q.clone().requires_grad_()), "gradient")
    refused(lib, lambda: call(q=q.float()), "q must be")
    refused(lib, lambda: call(q=q[:7]), "q must be")
    refused(lib, lambda: call(q=q[:, :31]), "q must be")
    out = torch.zeros(8, 16, 128, dtype=torch.bfloat16)
    refused(lib, lambda: call(out=out.half()), "one type")
    refused(lib, lambda: call(out=out[..., :64]), "out must be")
    refused(lib, lambda: call(out=out[:, :15]), "out must be")
    refused(lib, lambda: call(out=torch.zeros(8, 32, 64, dtype=torch.bfloat16)), "out must be")
    refused(lib, lambda: call(lse=torch.zeros(8, 16)), "lse must be")
    for kw in (dict(heads=3), dict(heads=1), dict(dim=256)):
        t2, cache2, step2, q2 = node(**kw)
        refused(lib, lambda: cache2.attend_diff(t2, step2, q2, lam), "pairs of heads")
    other = node(pages=201)
    refused(lib, lambda: cache.attend_diff(other[0], step, q, lam), "configuration")
    refused(lib, lambda: cache.attend_diff(t, other[2], q, lam), "configuration")
    with torch.no_grad():
        call(lam=lam.clone().requires_grad_(), weight=weight)
    call(out=out, lse=torch.zeros(8, 32))
    assert call().shape == (8, 16, 128) and lib.calls[-3:] == ["diff"] * 3


def test_strides_of_lambda_reach_the_library(lib):
    t, cache, step, q = node()
    for lam, token, head in ((torch.zeros(16), 0, 1), (torch.zeros(8, 16), 16, 1), (torch.zeros(16, 9).t(), 1, 9),
                             (torch.zeros(1, 16).expand(8, 16), 0, 1), (torch.zeros(8, 1).expand(8, 16), 1, 0)):
        cache.attend_diff(t, step, q, lam, weight=torch.zeros(128), gain=0.25, eps=0.5)
        d = lib.args[-1][10]._obj
        assert (d.lambda_token, d.lambda_head, d.gain, d.eps) == (token, head, 0.25, 0.5) and d.lambda_ == lam.data_ptr()


def test_the_workspace_fits_the_largest_layer(lib):
    t, cache, step, q = node(dim=128)
    small = KvCache(kv_config(**BASE))
    small.attend_diff(t, step, torch.zeros(8, 32, 64, dtype=torch.bfloat16), torch.zeros(16))
    first = step._diff_works[-1]
    cache.attend_diff(t, step, q, torch.zeros(16))
    assert len(step._diff_works) == 2 and step._diff_works[0] is first
    small.attend_diff(t, step, torch.zeros(8, 32, 64, dtype=torch.bfloat16), torch.zeros(16))
    assert lib.args[-1][-3] == step._diff_works[1].data_ptr() and len(step._diff_works) == 2


P, BIG = ctypes.c_void_p(0x100000), 1 << 40


def test_c_calls_reject_before_launch():
    lib, E = load(), L.AGFT_E_INVAL
    good = kv_config(**BASE)
    dense = lambda data=0x200000, token=2048, head=128, type_=L.AGFT_KV_BF16: L.agft_kv_dense(data, token, head, type_)  # noqa: E731
    args = lambda **kw: L.agft_diff_args(**{**dict(lambda_=0x300000, lambda_token=0, lambda_head=1, weight=None, eps=1e-5,  # noqa: E731
                                                   gain=1.0), **kw})

    def call(cfg=good, cache=P, cache_bytes=BIG, tables=P, step=P, tokens=9, new=1, q=dense(), diff=args(), out=dense(),
             lse=None, scale=1.0, work=P, work_bytes=BIG):
        ref = lambda x: None if x is None else ctypes.byref(x)                            # noqa: E731
        return lib.agft_diff_attend(ref(cfg), cache, cache_bytes, tables, BIG, step, BIG, tokens, new, ref(q), ref(diff),
                                    ref(out), lse, scale, work, work_bytes, None)
    nan, inf = float("nan"), float("inf")
    for kw in (dict(cfg=None), dict(cache=None), dict(cache_bytes=100), dict(tables=None), dict(step=None), dict(tokens=0),
               dict(new=0), dict(new=10), dict(q=None), dict(out=None), dict(diff=None), dict(work=None), dict(work_bytes=100),
               dict(scale=nan), dict(scale=inf), dict(lse=ctypes.c_void_p(0x200002)), dict(q=dense(type_=2), out=dense(type_=2)),
               dict(q=dense(type_=1)), dict(out=dense(token=0)), dict(out=dense(head=0)), dict(q=dense(data=0x200008)),
               dict(diff=args(lambda_=None)), dict(diff=args(lambda_=0x300002)), dict(diff=args(lambda_token=-1)),
               dict(diff=args(lambda_head=-1)), dict(diff=args(weight=0x300004)), dict(diff=args(eps=-1.0)),
               dict(diff=args(eps=nan)), dict(diff=args(gain=inf)), dict(cfg=kv_config(**{**BASE, "heads": 5}))):
        assert call(**kw) == E, kw
    assert call(cfg=kv_config(**{**BASE, "dim": 256})) == L.AGFT_E_UNSUPPORTED
    assert call(cfg=kv_config(**{**BASE, "dim": 96})) == L.AGFT_E_UNSUPPORTED
    for kw in (dict(heads=5), dict(dim=256), dict(dim=96), dict(pages=0)):
        assert lib.agft_diff_attend_bytes(ctypes.byref(kv_config(**{**BASE, **kw})), 9) == 0
    assert lib.agft_diff_attend_bytes(ctypes.byref(good), 0) == 0
    assert lib.agft_diff_attend_bytes(ctypes.byref(good), 1) <= lib.agft_diff_attend_bytes(ctypes.byref(good), 1 << 30)


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not found")
def test_no_kernel_spills(tmp_path):
    flags = [f for f in _build.HIPCC_FLAGS if f != "-shared"]
    out = subprocess.run([HIPCC, *flags, "--cuda-device-only", "-c", "-I", _build.INCLUDE,
                          os.path.join(_build.CSRC, "agft_diff.hip"), "-o", str(tmp_path / "diff.o"),
                          "-Rpass-analysis=kernel-resource-usage"], capture_output=True, text=True, check=True).stderr
    kernels = re.findall(r"Function Name: (\S+)(.*?)(?=Function Name:|\Z)", out, re.S)
    assert len(kernels) >= 16
    for name, body in kernels:
        scratch, vector = (int(re.search(p + r": (\d+)", body).group(1)) for p in (r"ScratchSize \[bytes/lane\]", "VGPRs Spill"))
        assert scratch == 0 and vector == 0, name


@pytest.mark.parametrize("form,dtype", [("e4m3", "bf16"), ("int8", "fp16")])
@pytest.mark.parametrize("norm", [False, True])
def test_the_bound_on_planted_mistakes(form, dtype, norm):
    """A rounded reference passes; a tenth of a number, swapped halves or a forgotten lambda do not."""
    w = Window([99, 700], [1, 3], 16, 4, 2, 64, form, dtype, 7, device="cpu")
    lam, weight = lambdas(w, True) * 0.4, weights(w) if norm else None
    out, lse, room, lse_room = reference(w, lam, weight, 0.3, 1e-5)
    assert bool(((out.to(w.dtype).double() - out).abs() <= room).all())
    assert bool(((lse.float().double() - lse).abs() <= lse_room).all())
    for spoil in (lambda y: y * torch.linspace(0.9, 1.1, 128, dtype=torch.float64), lambda y: y.roll(64, 1)):
        wrong = reference(w, lam, weight, 0.3, 1e-5, spoil)[0]
        assert bool(((wrong - out).abs() / room).amax(-1).min() > 1)
    wrong = reference(w, lam * 0.9, weight, 0.3, 1e-5)[0]
    assert norm or bool(((wrong - out).abs() / room).amax(-1).median() > 1)

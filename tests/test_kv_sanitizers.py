"""The cache's host code under the address and undefined-behaviour sanitizers
(CPU): compiled with hipcc, the sanitizers on its host pass only, and called by
tests/sanitize/kv_driver.c.  GPU code is not instrumented."""
import os

import pytest

import test_sanitizers as base
from paper_2508_01744_amd import _build


@pytest.mark.skipif(not os.path.exists(base.HIPCC) or not os.path.exists(base.CLANG), reason="hipcc or clang not found")
def test_cache_host_side_under_sanitizers(tmp_path):
    lib = str(tmp_path / "libkv_san.so")
    sources = [s for s in _build.SOURCES if "agft_kv" in s]
    assert len(sources) == 2
    base.subprocess.run([base.HIPCC, "--offload-arch=gfx950", "-O1", "-std=c++17", "-fPIC", "-shared", "-w",
                         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
                         "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
                         "-Xarch_host", "-fno-omit-frame-pointer", "-I", _build.INCLUDE, *sources, "-o", lib], check=True)
    exe = str(tmp_path / "kv_driver")
    base.subprocess.run([base.CLANG, "-std=c11", "-O1", "-g", "-fsanitize=address,undefined", "-fno-omit-frame-pointer",
                         "-D__HIP_PLATFORM_AMD__", "-I", _build.INCLUDE, "-I", os.path.join(base.ROCM, "include"),
                         os.path.join(base.SAN, "kv_driver.c"), lib, "-Wl,-rpath," + str(tmp_path), "-o", exe], check=True)
    out = base._run_clean(exe, {"ASAN_OPTIONS": "detect_leaks=0"})
    assert "0 failures" in out

"""The cache's kernels at build and launch (CPU): none of them spills registers,
and the driver in tests/c_abi/kv_launches.c, which stands in for the HIP
runtime's launch calls, sees the launches it expects."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2508_01744_amd import _build

HERE = os.path.dirname(os.path.abspath(__file__))
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")
HIPCC = os.environ.get("HIPCC", os.path.join(ROCM, "bin", "hipcc"))


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not found")
@pytest.mark.parametrize("name,kinds", [
    ("agft_kv.hip", dict(plan=1, plan_sums=1, plan_slots=1, reset=1, commit=1, append=18, export=18)),
    ("agft_kv_attend.hip", dict(few=12, tile=12))])
def test_no_kernel_spills(tmp_path, name, kinds):
    flags = [f for f in _build.HIPCC_FLAGS if f != "-shared"]
    cmd = [HIPCC, *flags, "--cuda-device-only", "-c", "-I", _build.INCLUDE, os.path.join(_build.CSRC, name), "-o",
           str(tmp_path / "kv.o"), "-Rpass-analysis=kernel-resource-usage"]
    out = subprocess.run(cmd, capture_output=True, text=True, check=True).stderr
    kernels = re.findall(r"Function Name: (\S+)(.*?)(?=Function Name:|\Z)", out, re.S)
    found = [re.search(r"detail\d+agft_kv_(\w+?)_kernel", n).group(1) for n, _ in kernels]
    assert {k: found.count(k) for k in set(found)} == kinds
    for n, body in kernels:
        scratch, vector = (int(re.search(p + r": (\d+)", body).group(1)) for p in (r"ScratchSize \[bytes/lane\]", "VGPRs Spill"))
        assert scratch == 0 and vector == 0, f"{n} spills {scratch} bytes per lane"


@pytest.mark.skipif(shutil.which("gcc") is None, reason="gcc not found")
def test_launches(tmp_path):
    assert os.path.exists(_build.LIB), "run __graft_entry__.build()"
    exe = str(tmp_path / "kv_launches")
    subprocess.run(["gcc", "-std=c11", "-O1", "-Wall", "-rdynamic", "-D__HIP_PLATFORM_AMD__", "-I", _build.INCLUDE,
                    "-I", os.path.join(ROCM, "include"), os.path.join(HERE, "c_abi", "kv_launches.c"), _build.LIB,
                    "-L", os.path.join(ROCM, "lib"), "-lamdhip64", "-Wl,-rpath," + os.path.dirname(_build.LIB),
                    "-Wl,-rpath," + os.path.join(ROCM, "lib"), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and "0 failures" in r.stdout, r.stdout[-4000:] + r.stderr[-2000:]

"""What sums of attention weight and evictions launch, without a GPU: the library's host sources with stand-ins for HIP
and the kernels."""
import os
import shutil
import subprocess

import pytest

from hostbuild import CSRC, ROCM, ROOT


def test_calls_launch_what_they_should(tmp_path):
    cxx = shutil.which("g++")
    if cxx is None or not os.path.exists(os.path.join(ROCM, "include", "hip", "hip_runtime.h")):
        pytest.skip("needs a host compiler and the HIP headers")
    exe = str(tmp_path / "launched_keep")
    src = [os.path.join(ROOT, "tests", "host", "launched_keep.cpp")]
    src += [os.path.join(CSRC, f) for f in ("api.cpp", "ops.cpp", "norm.cpp", "keep.cpp", "logprob.cpp", "planner.cpp",
                                            "locality.cpp")]
    r = subprocess.run([cxx, "-std=c++17", "-O1", "-w", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROCM, "include"),
                        "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-o", exe, *src],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and "FAILED" not in r.stdout and r.stdout.endswith("ok\n"), r.stdout[-4000:] + r.stderr[-1000:]

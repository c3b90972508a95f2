"""Build and run a program of tests/host: the library's host sources with tests/host/host_runtime.hpp in place of the
HIP runtime and the kernels."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2606_13097_amd", "csrc")
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")


def run(name: str, tmp_path, timeout: int = 120) -> str:
    cxx = shutil.which("g++")
    if cxx is None or not os.path.exists(os.path.join(ROCM, "include", "hip", "hip_runtime.h")):
        pytest.skip("needs a host compiler and the HIP headers")
    exe = str(tmp_path / name)
    src = [os.path.join(ROOT, "tests", "host", name + ".cpp")]
    src += [os.path.join(CSRC, f) for f in ("api.cpp", "ops.cpp", "planner.cpp", "locality.cpp")]
    r = subprocess.run([cxx, "-std=c++17", "-O1", "-w", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROCM, "include"),
                        "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-o", exe, *src],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=timeout)
    assert r.returncode == 0, f"exit {r.returncode}\n{r.stdout[-4000:]}\n{r.stderr[-1000:]}"
    return r.stdout

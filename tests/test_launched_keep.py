"""What sums of attention weight and evictions launch, without a GPU: the library's host sources with stand-ins for HIP
and the kernels."""
import os
import shutil
import subprocess

import pytest

from hostbuild import CSRC, ROCM, ROOT
from test_gpu_weights_plans import BLOCKS_OF_256, SHAPES_OF_256


@pytest.fixture(scope="module")
def exe(tmp_path_factory):
    cxx = shutil.which("g++")
    if cxx is None or not os.path.exists(os.path.join(ROCM, "include", "hip", "hip_runtime.h")):
        pytest.skip("needs a host compiler and the HIP headers")
    exe = str(tmp_path_factory.mktemp("host") / "launched_keep")
    src = [os.path.join(ROOT, "tests", "host", "launched_keep.cpp")]
    src += [os.path.join(CSRC, f) for f in ("api.cpp", "ops.cpp", "norm.cpp", "keep.cpp", "logprob.cpp", "planner.cpp",
                                            "locality.cpp")]
    r = subprocess.run([cxx, "-std=c++17", "-O1", "-w", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROCM, "include"),
                        "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-o", exe, *src],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    return exe


def run(*command):
    r = subprocess.run(command, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "FAILED" not in r.stdout, r.stdout[-4000:] + r.stderr[-1000:]
    return r.stdout


def test_calls_launch_what_they_should(exe):
    assert run(exe).endswith("ok\n")


def test_which_calls_have_blocks_of_256_keys(exe, tmp_path):
    """The GPU tests of blocks of 256 keys are of such blocks, by value and uploaded, with rows split; fp32 heads of 128
    have none."""
    lines, want = [], []
    for dtype, hq, hkv, d in SHAPES_OF_256 + [("f32", 64, 4, 128)]:
        for P, lens, toks, by_value in BLOCKS_OF_256.values():
            seq = [s for s, t in enumerate(toks) for _ in t]
            pos = [P + p for t in toks for p in t]
            head = (0 if dtype == "f32" else 1, hq, hkv, d, 16, P, len(lens), len(seq))
            lines.append(" ".join(map(str, (*head, *lens, *seq, *pos))))
            want.append((128 if (dtype, d) == ("f32", 128) else 256, int(by_value)))
    path = tmp_path / "calls"
    path.write_text("\n".join(lines))
    got = [tuple(map(int, line.split()[1:])) for line in run(exe, str(path)).splitlines()]
    assert [g[:2] for g in got] == want
    assert any(g[2] for g in got if g[0] == 256)

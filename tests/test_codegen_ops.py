"""The kernels of rotary forms, appending and prefix attention use no scratch memory: a tile or a row of theirs that
does not fit its registers would go through it on every step (the 256-row attention blocks once spilled hundreds of
registers to it, from an unrolled loop with several ways out)."""
import os
import tempfile

import pytest

from test_codegen import LIB, TOOLS, _code_objects, _private_sizes

KERNELS = {"rope_rows_kernel": 40, "prefix_attend_kernel": 16, "prefix_attend_f32_kernel": 8, "prefix_merge_kernel": 8,
           "graft_kernel": 48}


def test_kernels_use_no_scratch():
    if not os.path.exists(LIB) or not all(os.path.exists(t) for t in TOOLS):
        pytest.skip("needs the built library and the compiler's tools")
    seen = dict.fromkeys(KERNELS, 0)
    with tempfile.TemporaryDirectory() as tmp:
        for co in _code_objects(tmp):
            for name, size in _private_sizes(co).items():
                for k in KERNELS:
                    if f"{len(k)}{k}" in name:
                        seen[k] += 1
                        assert size == 0, f"{name}: {size} bytes of scratch a lane"
    assert seen == KERNELS      # every variant was found

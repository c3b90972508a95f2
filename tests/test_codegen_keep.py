"""The kernels of norms, of what a cache keeps of its positions and of log probabilities use no scratch memory (64
alternatives kept in 8 vectors a thread once spilled a log probability row's registers to it), and every variant that a
call can reach is there."""
import os
import tempfile

import pytest

from test_codegen import LIB, TOOLS, _code_objects, _private_sizes

KERNELS = {"norm_rope_kernel": 40, "norm_rope_grad_kernel": 8, "norm_weight_sum_kernel": 1, "attend_weights_kernel": 28,
           "weights_merge_kernel": 2, "evict_select_kernel": 3, "evict_copy_kernel": 16, "evict_inplace_kernel": 16,
           "logprob_kernel": 8, "logprob_merge_kernel": 2, "logprob_grad_kernel": 2}


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

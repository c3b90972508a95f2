"""Attention weight per cached position on the GPU, for plans that take several launches."""
import math

import numpy as np
import pytest
import torch

from opsutil import cache_memory, randn
from paper_2606_13097_amd import fcg
from test_gpu_weights import check

pytestmark = pytest.mark.gpu


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def test_splits_in_more_than_one_launch():
    """65530 sequences of one token and one of 2000, whose rows are split: more items than a launch takes.  A call with
    other queries runs before, so that the workspace holds other partials."""
    print("[gpu] more items than a launch takes", flush=True)
    singles, own, hq, d, T = 65530, 2000, 16, 64, 2048
    n = singles + own
    c = fcg.Cache(fcg.model_desc(1, hq, 1, d, 1e4, "bf16"), singles + 1, T, 16, singles + T // 16)
    mem = cache_memory(c, "bf16")[0]
    mem.fill_(float("nan"))
    seq = np.concatenate([np.arange(singles), np.full(own, singles)]).astype(np.int32)
    pos = np.concatenate([np.zeros(singles), np.arange(own)]).astype(np.int32)
    k = randn(gen(1), n, 1, d)
    fcg.fcg_append(c, 0, seq, pos)
    first, row = (fcg.fcg_cache_export_layout(c, s, 0)[0] for s in (0, singles))
    assert first[0] == 0 and row[0] == singles          # pages in the order of the sequences
    mem[0, :singles, 0, 0] = k[:singles, 0]
    at = torch.as_tensor(row.astype(np.int64), device="cuda")[torch.arange(own, device="cuda") // 16]
    mem[0, at, 0, torch.arange(own, device="cuda") % 16] = k[singles:, 0]

    def reference(q):
        """-> sums of the single positions, of the long sequence's, lse, the largest sum |q k| / sqrt(d)"""
        q64, k64 = q.double(), k[:, 0].double()
        z1 = (q64[:singles] * k64[:singles, None]).sum(-1) / math.sqrt(d)
        reach = float((q64[:singles].abs() * k64[:singles, None].abs()).sum(-1).max()) / math.sqrt(d)
        lse = torch.empty(n, hq, dtype=torch.float64, device="cuda")
        lse[:singles] = z1 + 0.25                       # (of more keys than these have: weights below 1)
        sums = torch.zeros(own, dtype=torch.float64, device="cuda")
        later = torch.ones(own, own, dtype=torch.bool, device="cuda").triu(1)
        for h in range(hq):
            z = q64[singles:, h] @ k64[singles:].T.contiguous() / math.sqrt(d)
            reach = max(reach, float((q64[singles:, h].abs() @ k64[singles:].abs().T.contiguous()).max()) / math.sqrt(d))
            z = z.masked_fill(later, -math.inf)
            lse[singles:, h] = torch.logsumexp(z, -1)
            sums += torch.softmax(z, -1).sum(0)
        return torch.exp(z1 - lse[:singles].float().double()).sum(-1), sums, lse.float(), reach

    for seed in (2, 3):
        q = randn(gen(seed), n, hq, d)
        one, long, lse, reach = reference(q)
        before = torch.zeros(singles + 1, 1, T, device="cuda")
        got, ref, attended = before.clone(), torch.zeros_like(before, dtype=torch.float64), torch.zeros_like(before, dtype=torch.bool)
        fcg.fcg_attend_weights(c, 0, -1, 0, seq, pos, q, lse, got)
        torch.cuda.synchronize()
        ref[:singles, 0, 0], ref[singles, 0, :own] = one, long
        attended[:singles, 0, 0] = attended[singles, 0, :own] = True
        check(got, before, ref, own * hq, reach, attended, d, f"queries {seed}")
    c.close()

"""Attention weight per cached position on the GPU, for plans that take several launches and for blocks of 256 keys."""
import math

import numpy as np
import pytest
import torch

from keeputil import fill_sequence
from opsutil import cache_memory, randn
from paper_2606_13097_amd import fcg
from test_gpu_weights import check, run_case

pytestmark = pytest.mark.gpu


# Calls with blocks of 256 keys (the prefix's positions, own positions and tokens' positions behind the prefix of each
# sequence; whether the plan goes by value): test_launched_keep.py holds them to that.
BLOCKS_OF_256 = {
    # an uploaded plan; a last block of keys of 208, a last tile of 16 rows, own blocks of few keys
    "list": (2000, [33] + [32] * 15, [list(range(33))] + [list(range(32))] * 15, False),
    # by value; a last block of 208 keys, tiles that see the prefix and a mask on the own keys
    "value": (8400, [2, 40] * 30, [[0, 1], [39, 5]] * 30, True),
    # one sequence, no prefix: tiles before, on and past the edge of each block
    "causal": (0, [1030], [list(range(1030))], False),
    # positions twice, tokens that see the prefix only, in any order
    "mixed": (1999, [300, 7], [list(range(0, 300, 2)) * 3, [-1] * 60 + [6, 3, 3]], False),
}
SHAPES_OF_256 = [("bf16", 64, 4, 128), ("bf16", 64, 4, 64), ("f32", 64, 4, 64)]


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


@pytest.mark.parametrize("dtype,hq,hkv,d", SHAPES_OF_256)
@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("case", list(BLOCKS_OF_256))
def test_blocks_of_256_keys_and_full_tiles(dtype, hq, hkv, d, page, case):
    print(f"[gpu] blocks of 256 keys, {case} {dtype} {d} page {page}", flush=True)
    P, lens, toks, _ = BLOCKS_OF_256[case]
    run_case(dtype, hq, hkv, d, page, P, lens, toks, flags=fcg.FCG_ADD if case == "value" else 0, shuffle=case == "mixed")


def test_weights_past_32_bits():
    """Weights of more than 2^31 bytes and a page table of many sequences: the last positions of the last sequence."""
    print("[gpu] weights past 2^31 bytes", flush=True)
    hq, hkv, d, T, S = 2, 2, 64, 1 << 20, 258
    c = fcg.Cache(fcg.model_desc(1, hq, hkv, d, 1e4, "bf16"), S, T, 16, T // 16 + 1)
    mem = cache_memory(c, "bf16")[0]
    x = randn(gen(1), T, hkv, d)
    fill_sequence(c, mem, 0, S - 1, 0, x)
    q = randn(gen(2), 1, hq, d)
    z = torch.stack([x[:, h].double() @ q[0, h].double() / math.sqrt(d) for h in range(hkv)])
    lse = torch.logsumexp(z, -1)
    w = torch.zeros(S, hkv, T, device="cuda")
    assert w.numel() * 4 > 1 << 31
    fcg.fcg_attend_weights(c, 0, 0, 0, [S - 1], [T - 1], q, lse.float()[None], w)
    torch.cuda.synchronize()
    reach = max(float((x[:, h].double().abs() @ q[0, h].double().abs()).max()) / math.sqrt(d) for h in range(hkv))
    attended = torch.ones(1, hkv, T, dtype=torch.bool, device="cuda")
    check(w[S - 1:], torch.zeros(1, hkv, T, device="cuda"), torch.exp(z - lse[:, None])[None], 1, reach, attended, d, "far weights")
    assert not bool(w[:S - 1].any())
    c.close()

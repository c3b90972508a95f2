"""Prefix attention on the GPU within bounds that count its roundings (opsbounds.py): the joined calls over what the cache
holds, long split prefixes, and every value row picked by some query."""
import numpy as np
import pytest
import torch

from opsbounds import check_attend_tight
from opsutil import DT, attend64, cache_memory, check_turned, freqs64, randn, rows_of, turn64
from paper_2606_13097_amd import fcg
from test_gpu_ops import Shared, bits, gen, make_rope, run_shared

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu(request):
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    print(f"[gpu] {request.node.name}", flush=True)


@pytest.mark.parametrize("dtype,page", [("bf16", 16), ("bf16", 0), ("f32", 16)])
def test_candidates_attend_over_what_is_stored(dtype, page):
    """Segments encoded, put into a library, stitched as the shared prefix of three candidates, which prefill, decode, retry
    in place and draft.  The rows that each call stores and the queries it encodes are held against the turn of what it was
    given, and the attention against those stored rows, so that no bound covers another's."""
    hq, hkv, d, L = 8, 2, 64, 2
    rope, w = make_rope(32, True, "parts", m=1.1)
    desc = fcg.model_desc(L, hq, hkv, d, 1e4, dtype)
    lens, dst, src = [150, 91], [91, 0], [40, 7]
    lib = fcg.Library(desc, sum(lens), 2)
    P = sum(lens)
    c = fcg.Cache(desc, 4, P + 80, page, 4 * (P + 80) // 16 if page else 0)
    mem = cache_memory(c, dtype)
    enc, val = [], []
    for i, n in enumerate(lens):
        k, v = randn(gen(i), L, n, hkv, d, dtype=dtype), randn(gen(9 + i), L, n, hkv, d, dtype=dtype)
        ke = torch.empty_like(k)
        fcg.fcg_rope_apply(rope, torch.arange(src[i], src[i] + n, dtype=torch.int32, device="cuda"), k=k, k_out=ke)
        torch.cuda.synchronize()
        check_turned(ke, turn64(k, np.arange(src[i], src[i] + n), w, True, 1.1), k, w, True, 1.1, dtype, f"segment {i}")
        fcg.fcg_lib_add_segment(lib, n, src[i], ke, v)
        enc.append(ke), val.append(v)
    fcg.fcg_graft_rope(c, lib, rope, [3, 3], [0, 1], dst)
    torch.cuda.synchronize()
    for i, n in enumerate(lens):
        at = np.arange(dst[i], dst[i] + n)
        for l in range(L):
            check_turned(rows_of(c, mem[0], l, 3, at), turn64(enc[i][l], np.full(n, dst[i] - src[i]), w, True), enc[i][l], w,
                         True, 1.0, dtype, f"grafted segment {i}")
            assert torch.equal(bits(rows_of(c, mem[1], l, 3, at).contiguous()), bits(val[i][l].contiguous()))
    end = {s: P for s in range(3)}

    def step(counts, seed, replace=False):
        seq = np.repeat(np.arange(3), counts)
        pos = np.concatenate([end[s] + np.arange(m) for s, m in enumerate(counts)])
        n = len(seq)
        x = randn(gen(seed), L, n, hq + 2 * hkv, d, dtype=dtype)
        for l in range(L):
            q, k, v = x[l, :, :hq], x[l, :, hq:hq + hkv], x[l, :, hq + hkv:]
            qe, out = (torch.empty((n, hq, d), dtype=DT[dtype], device="cuda") for _ in range(2))
            lse = torch.empty((n, hq), device="cuda")
            fcg.fcg_append(c, l, seq, pos, k, v, rope=rope, q=q, q_out=qe, flags=fcg.FCG_REPLACE if replace else 0)
            fcg.fcg_prefix_attend(c, l, 3, P, seq, pos, qe, out, lse)
            torch.cuda.synchronize()
            check_turned(qe, turn64(q, pos, w, True, 1.1), q, w, True, 1.1, dtype, "queries")
            for s in range(3):
                i = torch.as_tensor(np.flatnonzero(seq == s), device="cuda")
                check_turned(rows_of(c, mem[0], l, s, pos[seq == s]), turn64(k[i], pos[seq == s], w, True, 1.1), k[i], w,
                             True, 1.1, dtype, f"keys of {s}")
                assert torch.equal(bits(rows_of(c, mem[1], l, s, pos[seq == s]).contiguous()), bits(v[i].contiguous()))
                own = np.arange(P, pos[seq == s][-1] + 1)
                K, V = (torch.cat([rows_of(c, m, l, 3, np.arange(P)), rows_of(c, m, l, s, own)]) for m in mem)
                check_attend_tight(out[i], lse[i], attend64(qe[i], K, V, pos[seq == s], P), dtype, len(K), d,
                                   f"layer {l}, sequence {s}")

    for counts, seed, replace, on in (([20, 33, 1], 100, False, True), ([1, 1, 1], 101, False, False),
                                      ([1, 1, 1], 102, True, True), ([4, 1, 2], 103, False, True)):
        step(counts, seed, replace)
        for s, m in enumerate(counts):
            end[s] += m if on else 0
    c.close(), lib.close()


@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("hq,hkv,d,n_seq,tokens,P", [
    (32, 8, 128, 64, 1, 4321),         # a decode step: shared rows in two blocks of 128, own keys narrow
    (64, 8, 128, 32, 4, 6007),         # drafts: blocks of 256 rows
    (32, 8, 128, 8, 70, 5003),         # prompts
    (16, 4, 64, 20, 1, 3001),
    (16, 1, 128, 1, 1, 8190)])         # one task alone
def test_norm_error_over_a_long_split_prefix(page, hq, hkv, d, n_seq, tokens, P):
    own = [tokens + (53 * i) % 200 for i in range(n_seq)]
    sh = Shared("bf16", hq, hkv, d, page, P, own, 61, shuffle=False)
    seq = np.repeat(np.arange(n_seq), tokens)
    pos = np.concatenate([P + n - tokens + np.arange(tokens) for n in own])
    q, out, lse = run_shared(sh, seq, pos, 9)
    at = np.unique(np.linspace(0, len(seq) - 1, 16).astype(int))
    for t in at:
        K, V = sh.joined(int(seq[t]))
        check_attend_tight(out[t:t + 1], lse[t:t + 1], attend64(q[t:t + 1], K, V, pos[t:t + 1], P), "bf16", len(K), d,
                           f"token {t}", spread=True)
    sh.cache.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("tokens", [1, 40, 900])
def test_every_key_can_be_picked(dtype, page, tokens):
    """Each query is 8 times the key of one position, whose score is then some 30 above all others (90 against 0 +- 8), so
    the result is that position's value, whatever block, tile and split it lies in."""
    hq, hkv, d, P = 4, 1, 128, 901
    own = [130, 77, 64]
    sh = Shared(dtype, hq, hkv, d, page, P, own, 71, shuffle=False)
    every = [(i % 3, p) for i, p in enumerate(range(P))] + [(s, p) for s, m in enumerate(own) for p in range(P, P + m)]
    for r in range(6 if tokens < 900 else 1):           # few tokens: other picks each time
        at = every if tokens == 900 else [every[(i * 97 + r * 331) % len(every)] for i in range(tokens)]
        q = torch.empty((len(at), hq, d), dtype=DT[dtype], device="cuda")
        want = torch.empty((len(at), d), dtype=DT[dtype], device="cuda")
        for i, (s, p) in enumerate(at):
            K, V = sh.kv[sh.pseq] if p < P else sh.kv[s]
            q[i] = K[p if p < P else p - P, 0] * 8
            want[i] = V[p if p < P else p - P, 0]
        seq, pos = np.array([s for s, _ in at]), np.array([P + own[s] - 1 for s, _ in at])
        out = torch.full_like(q, float("nan"))
        fcg.fcg_prefix_attend(sh.cache, 1, sh.pseq, P, seq, pos, q, out)
        torch.cuda.synchronize()
        # bf16: the probability's rounding and the result's; the other keys have 1e-12 of the weight
        tol = (2.1 * 2.0 ** -8 if dtype == "bf16" else 2.0 ** -20) * want.double().abs()[:, None] + 1e-6
        err = (out.double() - want.double()[:, None]).abs()
        bad = (err > tol).any(-1).any(-1).nonzero().flatten().tolist()
        assert not bad, [at[i] for i in bad[:5]]
    sh.cache.close()

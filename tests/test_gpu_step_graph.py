"""A decode step of the calls together, captured: append with norms, attention over a shared prefix, the weights it puts
on the positions, log probabilities.  Two such graphs share the cache's workspace and are replayed in turn."""
import numpy as np
import pytest
import torch

from opsutil import cache_memory, randn
from paper_2606_13097_amd import fcg

pytestmark = pytest.mark.gpu


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


@pytest.mark.parametrize("page", [0, 16])
def test_captured_steps_give_what_eager_ones_give(page):
    print(f"[gpu] step graph, page {page}", flush=True)
    hq, hkv, d, n, prefix, vocab, top = 32, 8, 128, 24, 1500, 20011, 7
    c = fcg.Cache(fcg.model_desc(1, hq, hkv, d, 1e6, "bf16"), n + 1, 1600, page, 200 if page else 0)
    for m in cache_memory(c, "bf16"):
        m.zero_()
    k0 = randn(gen(1), prefix, hkv, d)
    fcg.fcg_append(c, 0, [n] * prefix, np.arange(prefix), k0, randn(gen(2), prefix, hkv, d))
    seq = np.arange(n, dtype=np.int32)
    for s in seq:                                  # three own positions of each sequence
        fcg.fcg_append(c, 0, [s] * 3, np.arange(prefix, prefix + 3), randn(gen(3), 3, hkv, d), randn(gen(4), 3, hkv, d))
    norm = fcg.Norm(randn(gen(5), d))
    q, k, v = (torch.empty(n, h, d, dtype=torch.bfloat16, device="cuda") for h in (hq, hkv, hkv))
    qe, out = torch.empty_like(q), torch.empty_like(q)
    lse, w = torch.empty(n, hq, device="cuda"), torch.empty(n + 1, hkv, 1600, device="cuda")
    logits = torch.empty(n, vocab, dtype=torch.bfloat16, device="cuda")
    target = torch.arange(n, dtype=torch.int32, device="cuda")
    lp, ent = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    ids, tlp = torch.empty(n, top, dtype=torch.int32, device="cuda"), torch.empty(n, top, device="cuda")
    ws = torch.empty(fcg.fcg_token_logprobs_workspace(n, vocab, top), dtype=torch.uint8, device="cuda")
    results = (qe, out, lse, w, lp, ent, ids, tlp)

    def step(own):
        pos = np.full(n, prefix + own, np.int32)
        fcg.fcg_append_norm(c, 0, seq, pos, k, v, norm, q=q, q_norm=norm, q_out=qe, flags=fcg.FCG_REPLACE)
        fcg.fcg_prefix_attend(c, 0, n, prefix, seq, pos, qe, out, lse)
        fcg.fcg_attend_weights(c, 0, n, prefix, seq, pos, qe, lse, w, flags=fcg.FCG_ADD)
        fcg.fcg_token_logprobs(logits, target, lp, ent, None, ids, tlp, ws)

    def inputs(seed):
        for i, t in enumerate((q, k, v, logits)):
            t.copy_(randn(gen(10 * seed + i), *t.shape))
        w.fill_(0.5)

    side, graphs = torch.cuda.Stream(), []
    inputs(0)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for own in (2, 1):
            step(own)
            side.synchronize()
            graphs.append(torch.cuda.CUDAGraph())
            with torch.cuda.graph(graphs[-1], stream=side):
                step(own)
    torch.cuda.synchronize()
    for seed in (1, 2, 3, 4):
        own = 2 if seed % 2 else 1
        inputs(seed)
        graphs[seed % 2 == 0].replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in results]
        inputs(seed)
        for t in results:
            if t is not w:
                t.zero_()
        step(own)
        torch.cuda.synchronize()
        for a, b in zip(got, results):
            assert torch.equal(a, b)
        assert bool(torch.isfinite(w).all()) and not bool((w[:n, :, :prefix] != 0.5).any())
        # every token puts weight 1 a query head on the positions it attends to (1600 sums rounded at 0.5, 96
        # rows of probabilities whose exponents are off by less than 2^-17: 8e-4)
        total = (w.double() - 0.5).sum((0, 2))
        assert float((total - n * (hq // hkv)).abs().max()) < 1e-2

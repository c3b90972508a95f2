"""Attention weight per cached position on the GPU, against the plain 64-bit form."""
import math

import numpy as np
import pytest
import torch

from keeputil import fill_sequence, weights64
from opsutil import cache_memory, randn
from paper_2606_13097_amd import fcg

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu(request):
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    print(f"[gpu] {request.node.name}", flush=True)


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def check(got, before, ref, rows, reach, attended, d, what):
    """A score is off by (d + 8) 2^-24 of sum |q k| / sqrt(d) (reach: the largest), its exponent and its probability by
    that, 2^-24 of |lse| + |score| in base 2 (3 |lse| + reach covers both) and 2^-22 for exp2 itself; the sum over `rows`
    rows by (rows + 16) 2^-24.  Positions that nothing attends to keep their bits."""
    share = (d + 8) * 2.0 ** -24 * reach + 4 * 2.0 ** -24 * (reach + 8) + 2.0 ** -22 + (rows + 16) * 2.0 ** -24
    assert torch.equal(got[~attended], before[~attended]), what
    err = (got.double() - ref).abs()[attended]
    assert bool((err <= share * ref[attended].abs() + 1e-30).all()), f"{what}: {float((err / ref[attended].abs()).max()):.3e}"


def setup(dtype, hq, hkv, d, page, P, lens, seed=1, layers=1, layer=0, scale=1.0):
    """A cache with a prefix of P positions in its last sequence and `lens[s]` own ones after it in sequence s."""
    n_seq = len(lens) + 1
    T = max([P, 1] + [P + n for n in lens])
    c = fcg.Cache(fcg.model_desc(layers, hq, hkv, d, 1e4, dtype), n_seq, T, page, n_seq * (T // 16 + 1) if page else 0)
    mem = cache_memory(c, dtype)[0]
    mem.fill_(float("nan"))            # what is not written is not read
    g = gen(seed)
    keys = [None] * n_seq
    for s, (a, n) in enumerate([(P, n) for n in lens] + [(0, P)]):
        x = randn(g, n, hkv, d, dtype=dtype, scale=scale)
        fill_sequence(c, mem, layer, s, a, x)
        keys[s] = x
    return c, keys, g


def run_case(dtype, hq, hkv, d, page, P, lens, toks, flags=0, scale=1.0, shuffle=False, twice=True):
    """toks[s]: positions (counted from P; -1: the prefix only) of the tokens of sequence s."""
    c, keys, g = setup(dtype, hq, hkv, d, page, P, lens, scale=scale)
    pre = len(lens)
    seq = np.concatenate([np.full(len(t), s) for s, t in enumerate(toks)]).astype(np.int32)
    pos = np.concatenate([np.asarray(t, dtype=np.int64) + P for t in toks]).astype(np.int32)
    if shuffle:
        order = np.random.default_rng(5).permutation(len(seq))
        seq, pos = seq[order], pos[order]
    q = randn(g, len(seq), hq, d, dtype=dtype)
    before = torch.rand(c.n_seqs, hkv, c.max_tokens, generator=g, device="cuda")
    ref, lse, rows, reach, attended = weights64(q, keys, pre, P, seq, pos, c.max_tokens, hkv)
    got = before.clone()
    lse32 = lse.float()
    fcg.fcg_attend_weights(c, 0, pre, P, seq, pos, q, lse32, got, flags=flags)
    torch.cuda.synchronize()
    if flags & fcg.FCG_ADD:
        ref = ref + before.double()
    check(got, before, ref, rows, reach, attended, d, f"{dtype} {hq}/{hkv} {d} P {P}")
    if twice:
        again = before.clone()
        fcg.fcg_attend_weights(c, 0, pre, P, seq, pos, q, lse32, again, flags=flags)
        assert torch.equal(again, got)
    c.close()


SHAPES = [("bf16", 32, 8, 128), ("bf16", 4, 4, 64), ("f32", 8, 2, 64), ("f32", 4, 2, 128), ("bf16", 16, 1, 128)]


@pytest.mark.parametrize("dtype,hq,hkv,d", SHAPES)
@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("P", [0, 1, 127, 129, 700])
def test_one_token_a_sequence(dtype, hq, hkv, d, page, P):
    lens = [1, 16, 17, 300, 128, 129]
    run_case(dtype, hq, hkv, d, page, P, lens, [[n - 1] for n in lens], flags=fcg.FCG_ADD)


@pytest.mark.parametrize("dtype,hq,hkv,d", SHAPES)
@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("P", [0, 333])
def test_several_tokens_a_sequence(dtype, hq, hkv, d, page, P):
    """Tokens in any order, the same position twice, tokens that see the prefix only, or nothing."""
    run_case(dtype, hq, hkv, d, page, P, [70, 200, 5], [[3, 3, 69, 40], list(range(100, 165)), [-1, 4]], shuffle=True)


@pytest.mark.parametrize("dtype,hq,hkv,d", SHAPES)
@pytest.mark.parametrize("P", [0, 64])
def test_more_tokens_and_sequences_than_go_by_value(dtype, hq, hkv, d, P):
    """An uploaded plan; few keys and many rows, so that rows are split and merged."""
    run_case(dtype, hq, hkv, d, 16, P, [40] * 70, [[39]] * 70)
    run_case(dtype, hq, hkv, d, 0, P, [700], [list(range(700))], flags=fcg.FCG_ADD)


@pytest.mark.parametrize("dtype,hq,hkv,d", SHAPES)
def test_splits_of_a_plan_by_value(dtype, hq, hkv, d):
    run_case(dtype, hq, hkv, d, 16, 200, [2] * 60, [[0, 1]] * 60)


def test_blocks_of_256_keys():
    run_case("bf16", 16, 8, 128, 16, 17000, [30, 300], [[29], [100, 299]])
    run_case("f32", 8, 8, 64, 0, 17001, [30], [[29, 28]])


def test_large_scores():
    """Peaked attention: most of a row's weight on one key."""
    run_case("bf16", 8, 2, 128, 0, 300, [100, 50], [[99, 20], [49]], scale=6.0)


@pytest.mark.parametrize("tokens", [1, 40])
def test_masked_and_unwritten_keys_do_not_leak(tokens):
    """Infinite and NaN keys behind a row's position leave its weights as they are; rows past the last token too."""
    c, keys, g = setup("bf16", 8, 2, 128, 0, 0, [300])
    mem = cache_memory(c, "bf16")[0]
    pos = np.arange(100, 100 + tokens).astype(np.int32)
    seq = np.zeros(tokens, np.int32)
    q = randn(g, tokens, 8, 128)
    _, lse, *_ = weights64(q, keys, 1, 0, seq, pos, c.max_tokens, 2)
    w = [torch.zeros(2, 2, c.max_tokens, device="cuda") for _ in range(2)]
    fcg.fcg_attend_weights(c, 0, 1, 0, seq, pos, q, lse.float(), w[0])
    mem[0, 0, :, 100 + tokens:200] = float("inf")
    mem[0, 0, :, 200:] = float("nan")
    fcg.fcg_attend_weights(c, 0, 1, 0, seq, pos, q, lse.float(), w[1])
    assert torch.equal(w[0], w[1]) and bool(torch.isfinite(w[0]).all()) and not bool(w[1][0, :, 100 + tokens:].any())
    mem[0, 0, 0, 100, 3] = float("-inf")       # a key that the last rows see: only its own sums change
    q[:, :, 3] = q[:, :, 3].abs() + 0.1
    fcg.fcg_attend_weights(c, 0, 1, 0, seq, pos, q, lse.float(), w[0])
    mem[0, 0, 0, 100, 3] = 0
    fcg.fcg_attend_weights(c, 0, 1, 0, seq, pos, q, lse.float(), w[1])
    other = torch.ones(c.max_tokens, dtype=torch.bool, device="cuda")
    other[100] = False
    assert torch.equal(w[0][0, :, other], w[1][0, :, other]) and float(w[0][0, 0, 100]) == 0.0


@pytest.mark.parametrize("page", [0, 16])
def test_sums_over_keys_are_the_rows(page):
    """After attention's own lse every row's weights add up to 1, over prefix and own keys, at a layer of several; query
    rows in strided slices that start at any element."""
    hq, hkv, d, P, L = 8, 2, 64, 500, 3
    c, keys, g = setup("bf16", hq, hkv, d, page, P, [60, 90], layers=L, layer=2)
    V = cache_memory(c, "bf16")[1]
    V.zero_()
    seq, pos = np.array([0, 1, 1], np.int32), np.array([P + 59, P + 89, P + 30], np.int32)
    flat = randn(g, 1 + 3 * (hq + 3) * d)
    q = flat[1:].view(3, hq + 3, d)[:, 2:hq + 2]
    out, lse = torch.empty(3, hq, d, dtype=torch.bfloat16, device="cuda"), torch.empty(3, hq, device="cuda")
    w = torch.zeros(3, hkv, c.max_tokens, device="cuda")
    fcg.fcg_prefix_attend(c, 2, 2, P, seq, pos, q, out, lse)
    fcg.fcg_attend_weights(c, 2, 2, P, seq, pos, q, lse, w, flags=fcg.FCG_ADD)
    total = w.double().sum((0, 2))
    assert bool((total - 3 * hq / hkv).abs().max() < 1e-4), total
    assert not bool(w[0, :, :P].any()) and not bool(w[2, :, P:].any())


def test_replays_in_a_graph_on_another_stream():
    hq, hkv, d, P = 16, 4, 128, 900
    lens = [20] * 10
    c, keys, g = setup("bf16", hq, hkv, d, 16, P, lens)
    seq = np.arange(10, dtype=np.int32)
    pos = np.full(10, P + 19, np.int32)
    q, out = randn(g, 10, hq, d), torch.empty(10, hq, d, dtype=torch.bfloat16, device="cuda")
    cache_memory(c, "bf16")[1].zero_()
    lse, w = torch.empty(10, hq, device="cuda"), torch.zeros(11, hkv, c.max_tokens, device="cuda")

    def step():
        fcg.fcg_prefix_attend(c, 0, 10, P, seq, pos, q, out, lse)
        fcg.fcg_attend_weights(c, 0, 10, P, seq, pos, q, lse, w, flags=fcg.FCG_ADD)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step()
    for seed in (1, 2, 3):
        q.copy_(randn(gen(seed), 10, hq, d))
        w.fill_(0.25)
        graph.replay()
        graph.replay()
        torch.cuda.synchronize()
        got = w.clone()
        w.fill_(0.25)
        step()
        step()
        torch.cuda.synchronize()
        assert torch.equal(got, w) and bool(torch.isfinite(w).all())


def test_captures_that_need_an_upload_or_a_workspace_are_refused():
    for n in (150, 100):       # more than 128 tokens; splits that have no workspace yet
        c, keys, g = setup("bf16", 8, 2, 64, 0, 0, [200])
        w = torch.zeros(2, 2, c.max_tokens, device="cuda")
        seq, pos = np.zeros(n, np.int32), np.full(n, 199, np.int32)
        q, lse = randn(g, n, 8, 64), torch.zeros(n, 8, device="cuda")
        graph, status = torch.cuda.CUDAGraph(), None
        with torch.cuda.graph(graph):
            try:
                fcg.fcg_attend_weights(c, 0, 1, 0, seq, pos, q, lse, w)
            except fcg.FcgError as e:
                status = e.status
            w.add_(1.0)
        assert status == fcg.FCG_ESTATE
        fcg.fcg_attend_weights(c, 0, 1, 0, seq, pos, q, lse, w)
        torch.cuda.synchronize()
        assert bool(w[0, :, :200].all())
        c.close()


def test_offsets_past_32_bits():
    """A cache of more than 2^32 elements and weights past 2^31 bytes: the last sequence's last positions."""
    hq, hkv, d, T, S = 2, 2, 128, 1 << 20, 17
    c = fcg.Cache(fcg.model_desc(1, hq, hkv, d, 1e4, "bf16"), S, T)
    mem = cache_memory(c, "bf16")[0]
    x = randn(gen(1), T, hkv, d)
    fill_sequence(c, mem, 0, S - 1, 0, x)
    q = randn(gen(2), 1, hq, d)
    z = torch.stack([x[:, h].double() @ q[0, h].double() / math.sqrt(d) for h in range(hkv)])
    lse = torch.logsumexp(z, -1)
    w = torch.zeros(S, hkv, T, device="cuda")
    fcg.fcg_attend_weights(c, 0, 0, 0, [S - 1], [T - 1], q, lse.float()[None], w)
    ref = torch.exp(z - lse[:, None])
    assert not bool(w[:S - 1].any())
    assert float((w[S - 1].double() - ref).norm() / ref.norm()) < 1e-5
    c.close()

"""Eviction by weight on the GPU, against the plain form."""
import numpy as np
import pytest
import torch

from keeputil import kept64
from opsutil import cache_memory, check_turned, freqs64, randn, rows_of, turn64
from paper_2606_13097_amd import fcg

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu(request):
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    print(f"[gpu] {request.node.name}", flush=True)


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def bits(t):
    return t.contiguous().view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32)


def rope_of(form, d):
    """(handle or None, frequencies, pairs): the cache's own form, a part of the head in halves or in pairs."""
    if form == "own":
        return None, freqs64(d, 1e4), False
    rot, pairs = {"half": (d - 16, False), "pairs": (d // 2, True), "whole": (d, True)}[form]
    return fcg.fcg_rope_create(rot, 1e4, layout=int(pairs), attn_factor=1.3), freqs64(rot, 1e4), pairs


def make(dtype, hkv, d, page, lens, L=2, spare=0, extra=0):
    n_seq = len(lens) + spare
    T = max(max(lens), 16) + extra
    pages = sum(-(-n // 16) for n in lens) + spare * -(-T // 16)
    c = fcg.Cache(fcg.model_desc(L, hkv * 2, hkv, d, 1e4, dtype), n_seq, T, page, pages if page else 0)
    mem = cache_memory(c, dtype)
    for m in mem:
        m.fill_(float("nan"))
    rows = []
    for s, n in enumerate(lens):
        pos = np.arange(n)
        if n:
            fcg.fcg_append(c, 0, np.full(n, s), pos, n_layers=L)
        kv = [randn(gen(10 * s + i), L, n, hkv, d, dtype=dtype) for i in (0, 1)]
        for m, x in zip(mem, kv):
            for l in range(L):
                if not n:
                    continue
                if page:
                    pt, _, _ = fcg.fcg_cache_export_layout(c, s, l)
                    m[l][torch.as_tensor(pt.astype(np.int64))[pos // 16], :, pos % 16] = x[l]
                else:
                    m[l, s, :, :n] = x[l].transpose(0, 1)
        rows.append(kv)
    return c, mem, rows


def weights_of(c, L, seed, ties=0.3):
    w = torch.rand(L, c.n_seqs, c.desc.n_kv_heads, c.max_tokens, generator=gen(seed), device="cuda")
    few = torch.round(w * 4) / 4           # many equal ones
    return torch.where(torch.rand(w.shape, generator=gen(seed + 1), device="cuda") < ties, few, w)


def check(c, mem, rows, w0, w, kept, src, dst, keep, first, recent, freqs, pairs, dtype, lens):
    L, hkv, d, T = c.desc.n_layers, c.desc.n_kv_heads, c.desc.head_dim, c.max_tokens
    w0n = w0.cpu().numpy()
    for i, (s, t, k) in enumerate(zip(src, dst, keep)):
        n = min(int(k), lens[s])
        _, length, written = fcg.fcg_cache_export_layout(c, int(t), 0)
        assert length == n and written[:n].all() and not written[n:].any()
        K, V = (torch.stack([rows_of(c, m, l, int(t), np.arange(n)) for l in range(L)]) for m in mem)
        for l in range(L):
            for h in range(hkv):
                at = kept64(w0n[l, s, h], lens[s], int(k), first, recent)
                ta = torch.as_tensor(at, device="cuda")
                assert len(at) == n
                if kept is not None:
                    assert torch.equal(kept[l, i, h, :n].long(), ta), f"item {i} layer {l} head {h}"
                    assert bool((kept[l, i, h, n:] == -7).all())
                want = torch.zeros(T, device="cuda")
                want[:n] = w0[l, s, h][ta]
                assert torch.equal(torch.nan_to_num(w[l, t, h], nan=-5.0), torch.nan_to_num(want, nan=-5.0))
                x = rows[s][0][l, ta, h][:, None]
                moved = np.arange(n) - at
                check_turned(K[l, :, h][:, None], turn64(x, moved, freqs, pairs), x, freqs, pairs, 1.0, dtype, f"keys {l} {h}")
                still = torch.as_tensor(moved == 0, device="cuda")
                assert torch.equal(bits(K[l, :, h][still]), bits(x[:, 0][still]))
                assert torch.equal(bits(V[l, :, h]), bits(rows[s][1][l, ta, h]))


@pytest.mark.parametrize("dtype,hkv,d", [("bf16", 8, 128), ("bf16", 1, 64), ("f32", 2, 64), ("f32", 2, 128)])
@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("form", ["own", "half", "pairs", "whole"])
def test_into_other_sequences_and_in_place(dtype, hkv, d, page, form):
    lens = [700, 1, 129, 64, 333]
    rope, freqs, pairs = rope_of(form, d)
    c, mem, rows = make(dtype, hkv, d, page, lens, spare=4, extra=9)
    w = weights_of(c, 2, 1)
    src, dst, keep = [0, 1, 2, 0, 3, 4], [5, 6, 2, 7, 3, 8], [200, 9, 65, 700, 64, 1]
    kept = torch.full((2, 6, hkv, 700), -7, dtype=torch.int32, device="cuda")
    w0 = w.clone()
    fcg.fcg_evict(c, src, dst, keep, w, first=4, recent=20, rope=rope, kept=kept)
    torch.cuda.synchronize()
    check(c, mem, rows, w0, w, kept, src, dst, keep, 4, 20, freqs, pairs, dtype, lens)
    for s in (0, 1, 4):       # the sources stay
        assert torch.equal(w[:, s], w0[:, s])
        got = [torch.stack([rows_of(c, m, l, s, np.arange(lens[s])) for l in range(2)]) for m in mem]
        assert all(torch.equal(bits(a), bits(b)) for a, b in zip(got, rows[s]))
    c.close()


@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("n,keep,first,recent", [(1000, 1000, 0, 0), (1000, 999, 0, 0), (1000, 1, 0, 0), (1000, 1, 5, 5),
                                                 (1000, 30, 20, 20), (1000, 30, 0, 30), (1000, 640, 600, 0), (2, 1, 0, 1),
                                                 (1000, 0, 3, 3), (1000, 500, 2000, 0), (1000, 128, 0, 0), (129, 128, 0, 0)])
def test_in_place_edges(page, n, keep, first, recent):
    c, mem, rows = make("bf16", 2, 128, page, [n], extra=40)
    w = weights_of(c, 2, 3)
    w0 = w.clone()
    kept = torch.full((2, 1, 2, keep), -7, dtype=torch.int32, device="cuda")
    fcg.fcg_evict(c, [0], [0], [keep], w, first=first, recent=recent, kept=kept)
    torch.cuda.synchronize()
    check(c, mem, rows, w0, w, kept, [0], [0], [keep], first, recent, freqs64(128, 1e4), False, "bf16", [n])
    c.close()


@pytest.mark.parametrize("in_place", [False, True])
def test_weights_of_every_kind(in_place):
    """Infinities, NaN, zeros of both signs, negative and subnormal weights, all equal ones."""
    n = 600
    c, mem, rows = make("bf16", 4, 64, 0, [n], L=2, spare=1)
    w = weights_of(c, 2, 5) - 0.5
    w[0, 0, 0, ::7] = float("inf")
    w[0, 0, 1, ::3] = float("nan")
    w[0, 0, 1, 1::3] = float("-inf")
    w[0, 0, 2] = 0.0
    w[0, 0, 2, ::2] = -0.0
    w[0, 0, 3] = float("nan")
    w[1, 0, 0] = 1e-42 * torch.arange(c.max_tokens, device="cuda")
    w[1, 0, 1] = -w[1, 0, 0]
    w[1, 0, 2] = 3.5
    w0 = w.clone()
    kept = torch.full((2, 1, 4, 400), -7, dtype=torch.int32, device="cuda")
    fcg.fcg_evict(c, [0], [0 if in_place else 1], [400], w, first=3, recent=8, kept=kept)
    torch.cuda.synchronize()
    check(c, mem, rows, w0, w, kept, [0], [0 if in_place else 1], [400], 3, 8, freqs64(64, 1e4), False, "bf16", [n])


@pytest.mark.parametrize("dst", [0, 1])
def test_rows_longer_than_the_registers_hold(dst):
    """Selection over several segments of 16384 weights, with a threshold shared by them; far moves."""
    n = 50000
    c, mem, rows = make("bf16", 1, 64, 16, [n], L=1, spare=1)
    w = weights_of(c, 1, 7, ties=0.9)
    w0 = w.clone()
    kept = torch.full((1, 1, 1, 20001), -7, dtype=torch.int32, device="cuda")
    rope, freqs, pairs = rope_of("whole", 64)
    fcg.fcg_evict(c, [0], [dst], [20001], w, first=100, recent=16400, rope=rope, kept=kept)
    torch.cuda.synchronize()
    check(c, mem, rows, w0, w, kept, [0], [dst], [20001], 100, 16400, freqs, pairs, "bf16", [n])
    c.close()


@pytest.mark.parametrize("n", [1024, 1025, 4096, 8192, 8193, 16384, 16385])
@pytest.mark.parametrize("dst", [0, 1])
def test_rows_at_the_sizes_of_the_blocks(n, dst):
    """The longest rows that a block of each size holds, and one position more; weights that share their upper bits."""
    c, mem, rows = make("f32", 2, 64, 0, [n], L=1, spare=1, extra=3)
    w = 1.0 + weights_of(c, 1, n) * 2.0 ** -12
    w0 = w.clone()
    keep = n // 3
    kept = torch.full((1, 1, 2, keep), -7, dtype=torch.int32, device="cuda")
    fcg.fcg_evict(c, [0], [dst], [keep], w, first=1, recent=5, kept=kept)
    torch.cuda.synchronize()
    check(c, mem, rows, w0, w, kept, [0], [dst], [keep], 1, 5, freqs64(64, 1e4), False, "f32", [n])
    c.close()


def test_more_items_than_a_launch_takes_and_no_list_of_positions():
    lens = [50 + 3 * i for i in range(150)]
    c, mem, rows = make("bf16", 2, 64, 16, lens, L=1)
    src = np.arange(150)
    keep = 10 + src % 30
    w = weights_of(c, 1, 9)
    w0 = w.clone()
    free = sum(-(-n // 16) for n in lens)
    fcg.fcg_evict(c, src, src, keep, w, recent=2)
    torch.cuda.synchronize()
    check(c, mem, rows, w0, w, None, src, src, keep, 0, 2, freqs64(64, 1e4), False, "bf16", lens)
    used = np.concatenate([fcg.fcg_cache_export_layout(c, s, 0)[0] for s in src])
    used = used[used >= 0]
    assert len(np.unique(used)) == len(used) == sum(-(-k // 16) for k in keep) < free


def test_values_read_from_the_library():
    """A source whose values lie in the library goes into another sequence; in place it is refused."""
    hkv, d, L = 2, 64, 2
    desc = fcg.model_desc(L, 4, hkv, d, 1e4, "bf16")
    lib = fcg.fcg_lib_create(desc, 200, 2)
    k, v = randn(gen(1), L, 100, hkv, d), randn(gen(2), L, 100, hkv, d)
    fcg.fcg_lib_add_segment(lib, 100, 0, k, v)
    c = fcg.Cache(desc, 2, 160, 16, 30, fcg.FCG_ALIAS_V)
    fcg.fcg_graft(c, lib, [0], [0], [0])
    w = weights_of(c, L, 11)
    w0 = w.clone()
    with pytest.raises(fcg.FcgError) as e:
        fcg.fcg_evict(c, [0], [0], [50], w)
    assert e.value.status == fcg.FCG_ESTATE and torch.equal(w, w0)
    kept = torch.full((L, 1, hkv, 50), -7, dtype=torch.int32, device="cuda")
    fcg.fcg_evict(c, [0], [1], [50], w, kept=kept)
    torch.cuda.synchronize()
    check(c, cache_memory(c, "bf16"), [[k, v]], w0, w, kept, [0], [1], [50], 0, 0, freqs64(d, 1e4), False, "bf16", [100])
    assert (fcg.fcg_cache_export_v_alias(c, 0)[:6] >= 0).all() and (fcg.fcg_cache_export_v_alias(c, 1) == -1).all()
    fcg.fcg_evict(c, [1], [1], [20], w)          # whose values are its own


@pytest.mark.parametrize("page", [0, 16])
def test_decode_with_scores_and_eviction(page):
    """As a program uses them: every step appends normalised keys, attends, keeps score; at its budget the sequence is
    squeezed and goes on.  Against the same steps by the plain forms on the rows the cache holds."""
    hq, hkv, d, budget = 8, 2, 64, 48
    rope, freqs, pairs = rope_of("pairs", d)
    c = fcg.Cache(fcg.model_desc(1, hq, hkv, d, 1e4, "f32"), 2, 80, page, 10 if page else 0)
    w = torch.zeros(1, 2, hkv, 80, device="cuda")
    norm = fcg.Norm(randn(gen(1), d, dtype="f32"), eps=1e-6)
    length, score = 0, torch.zeros(hkv, 0, dtype=torch.float64, device="cuda")
    mem = cache_memory(c, "f32")
    for step in range(120):
        q, k, v = (randn(gen(100 * step + i), 1, h, d, dtype="f32") for i, h in ((0, hq), (1, hkv), (2, hkv)))
        qe, out, lse = torch.empty_like(q), torch.empty_like(q), torch.empty(1, hq, device="cuda")
        fcg.fcg_append_norm(c, 0, [0], [length], k, v, norm, rope=rope, q=q, q_norm=norm, q_out=qe)
        fcg.fcg_prefix_attend(c, 0, 0, 0, [0], [length], qe, out, lse)
        fcg.fcg_attend_weights(c, 0, 0, 0, [0], [length], qe, lse, w[0], flags=fcg.FCG_ADD)
        length += 1
        K, V = (rows_of(c, m, 0, 0, np.arange(length)).double() for m in mem)
        z = torch.einsum("hgd,nhd->hgn", qe[0].double().view(hkv, hq // hkv, d).cpu(), K.cpu()) / d ** 0.5
        p = torch.softmax(z, -1).cuda()
        o = torch.einsum("hgn,nhd->hgd", p.cpu(), V.cpu()).reshape(hq, d)
        assert float((out[0].double().cpu() - o).abs().max()) < 1e-5
        score = torch.cat([score, torch.zeros(hkv, 1, dtype=torch.float64, device="cuda")], 1) + p.sum(1)
        assert float((w[0, 0, :, :length].double() - score).abs().max()) < 1e-4 and not bool(w[0, 0, :, length:].any())
        if length == 64:
            kept = torch.empty(1, 1, hkv, budget, dtype=torch.int32, device="cuda")
            before = w.clone()
            fcg.fcg_evict(c, [0], [0], [budget], w, first=2, recent=8, rope=rope, kept=kept)
            for h in range(hkv):
                at = kept64(before[0, 0, h].cpu().numpy(), 64, budget, 2, 8)
                assert np.array_equal(kept[0, 0, h].cpu().numpy(), at)
            score = torch.gather(score, 1, kept[0, 0].long())
            length = budget
    assert fcg.fcg_cache_export_layout(c, 0, 0)[1] == length


def test_replays_in_a_graph_on_another_stream():
    c, mem, rows = make("bf16", 4, 128, 0, [500, 300], spare=2)
    rope, freqs, pairs = rope_of("half", 128)
    w = weights_of(c, 2, 13)
    kept = torch.full((2, 2, 4, 200), -7, dtype=torch.int32, device="cuda")
    args = dict(first=4, recent=16, rope=rope, kept=kept)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        fcg.fcg_evict(c, [0, 1], [2, 3], [200, 100], w, **args)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            fcg.fcg_evict(c, [0, 1], [2, 3], [200, 100], w, **args)
    for seed in (1, 2, 3):
        w.copy_(weights_of(c, 2, seed))
        for m in mem:
            m[:, 2:] = float("nan")
        kept.fill_(-7)
        graph.replay()
        torch.cuda.synchronize()
        check(c, mem, rows, weights_of(c, 2, seed), w, kept, [0, 1], [2, 3], [200, 100], 4, 16, freqs, pairs, "bf16",
              [500, 300])
    paged, _, _ = make("bf16", 2, 64, 16, [100], spare=1)
    status, w = None, weights_of(paged, 2, 1)
    with torch.cuda.graph(torch.cuda.CUDAGraph()):
        try:
            fcg.fcg_evict(paged, [0], [1], [50], w)
        except fcg.FcgError as e:
            status = e.status
        w.add_(1.0)
    assert status == fcg.FCG_ESTATE and fcg.fcg_cache_export_layout(paged, 1, 0)[1] == 0

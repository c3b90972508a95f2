"""Norms of queries and keys with their turn on the GPU, their gradient and appending, against plain 64-bit forms."""
import numpy as np
import pytest
import torch

from normutil import check_grad, check_normed, grad64, weights64
from opsutil import DT, HALF_STEP, cache_memory, freqs64, randn, rows_of
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


def dpos(pos):
    return torch.as_tensor(pos, dtype=torch.int32, device="cuda")


def make_rope(rot, pairs, m=1.0, theta=1e4):
    return fcg.fcg_rope_create(rot, theta, layout=int(pairs), attn_factor=m), freqs64(rot, theta)


def make_weight(g, kind, layers, heads, d, dtype):
    shape = {"none": None, "one": (d,), "heads": (heads, d), "layers": (layers, 1, d), "all": (layers, heads, d)}[kind]
    return None if shape is None else randn(g, *shape, dtype=dtype, scale=0.5)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("d,rot", [(128, 128), (128, 48), (64, 64), (64, 16)])
def test_apply_all_forms(dtype, pairs, d, rot):
    for kind, offset, m, n, layers, hq, hk in (("one", 0.0, 1.0, 1, 1, 4, 1), ("all", 1.0, 1.25, 77, 3, 5, 2),
                                               ("heads", 0.0, 0.5, 300, 1, 1, 0), ("layers", 1.0, 1.0, 700, 2, 8, 8),
                                               ("none", 0.0, 1.0, 33, 9, 4, 4)):
        g = gen(rot + n)
        rope, w = make_rope(rot, pairs, m)
        pos = np.random.default_rng(n).integers(0, 50000, n)
        q, k = randn(g, layers, n, hq, d, dtype=dtype, scale=3.0), randn(g, layers, n, hk, d, dtype=dtype, scale=0.01)
        qo, ko = torch.full_like(q, float("nan")), torch.full_like(k, float("nan"))
        qw, kw = make_weight(g, kind, layers, hq, d, dtype), make_weight(g, kind, layers, max(hk, 1), d, dtype)
        qn, kn = fcg.Norm(qw, 1e-6, offset), fcg.Norm(kw, 1e-3, offset)
        fcg.fcg_norm_rope_apply(rope, dpos(pos), q, qn, qo, *((k, kn, ko) if hk else ()))
        torch.cuda.synchronize()
        check_normed(qo, q, weights64(qw, offset, layers, hq, d), 1e-6, pos, w, pairs, m, dtype, f"q {kind}")
        if hk:
            check_normed(ko, k, weights64(kw, offset, layers, hk, d), 1e-3, pos, w, pairs, m, dtype, f"k {kind}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("start", [0, 1, 3])
def test_slices_any_start_one_side_turned_only_in_place(dtype, start):
    """q and k as slices of a fused projection at any element, a weight that starts at any element; q normalised, k
    turned only (the bits of the turn alone); then in place."""
    n, hq, hk, d = 37, 6, 2, 64
    rope, w = make_rope(48, True, 1.5)
    flat = randn(gen(start), start + n * (hq + 2 * hk) * d + 5, dtype=dtype)
    x = flat[start:start + n * (hq + 2 * hk) * d].view(n, hq + 2 * hk, d)
    weight = randn(gen(9), hq * d + start, dtype=dtype)[start:].view(hq, d)
    pos = np.arange(1000, 1000 + n)
    out, turned = torch.empty((2, n, hq + hk, d), dtype=DT[dtype], device="cuda")
    norm = fcg.Norm(weight)
    was = x.clone()
    fcg.fcg_norm_rope_apply(rope, dpos(pos), x[:, :hq], norm, out[:, hk:], x[:, hq:hq + hk], None, out[:, :hk])
    fcg.fcg_rope_apply(rope, dpos(pos), k=x[:, hq:hq + hk], k_out=turned[:, :hk])
    fcg.fcg_norm_rope_apply(rope, dpos(pos), x[:, :hq], norm, x[:, :hq], x[:, hq:hq + hk], None, x[:, hq:hq + hk])
    torch.cuda.synchronize()
    check_normed(out[:, hk:][None], was[:, :hq][None], weights64(weight, 0.0, 1, hq, d), 1e-6, pos, w, True, 1.5, dtype, "q")
    assert torch.equal(bits(out[:, :hk]), bits(turned[:, :hk]))
    assert torch.equal(bits(x[:, :hq]), bits(out[:, hk:])) and torch.equal(bits(x[:, hq:hq + hk]), bits(out[:, :hk]))
    assert torch.equal(bits(x[:, hq + hk:]), bits(was[:, hq + hk:]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_of_zeros_large_and_not_finite(dtype):
    """Zero rows give zeros, large and small ones keep their accuracy, an infinity or NaN stays in its row."""
    d, n = 128, 6
    rope, w = make_rope(128, False)
    x = randn(gen(1), 1, n, 2, d, dtype=dtype)
    x[0, 0] = 0
    x[0, 1] *= 1e15
    x[0, 2] *= 1e-15
    x[0, 3, 0, 5] = float("inf")
    x[0, 4, 1, 7] = float("nan")
    y = torch.empty_like(x)
    fcg.fcg_norm_rope_apply(rope, dpos(range(n)), x, fcg.Norm(None, 1e-30), y)
    dx = torch.empty_like(x)
    fcg.fcg_norm_rope_backward(rope, dpos(range(n)), x, fcg.Norm(None, 1e-30), torch.ones_like(x), dx)
    torch.cuda.synchronize()
    ok = torch.ones(n, 2, dtype=torch.bool)
    ok[3, 0] = ok[4, 1] = False
    for r, (a, b) in enumerate(ok.tolist()):
        for h, fine in enumerate((a, b)):
            assert bool(torch.isfinite(y[0, r, h].float()).all()) == fine and bool(torch.isfinite(dx[0, r, h].float()).all()) == fine
    assert not bool(y[0, 0].any())
    xs = torch.where(ok[None, :, :, None].cuda(), x, torch.ones_like(x))
    ys = torch.where(ok[None, :, :, None].cuda(), y, torch.zeros_like(y))
    ys[~ok[None].cuda()] = 0
    for r in (0, 1, 2, 5):
        check_normed(ys[:, r:r + 1], xs[:, r:r + 1], weights64(None, 0, 1, 2, d), 1e-30, [r], w, False, 1.0, dtype, f"row {r}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("d,rot", [(128, 128), (128, 48), (64, 64), (64, 16)])
def test_gradient_all_forms(dtype, pairs, d, rot):
    for kind, offset, m, n, layers, hq, hk in (("one", 0.0, 1.0, 1, 1, 4, 1), ("all", 1.0, 1.25, 77, 3, 5, 2),
                                               ("heads", 0.0, 0.5, 301, 1, 17, 0), ("layers", 1.0, 1.0, 65, 2, 24, 8),
                                               ("none", 0.0, 1.0, 33, 9, 4, 4)):
        g = gen(rot + n)
        rope, w = make_rope(rot, pairs, m)
        pos = np.random.default_rng(n).integers(0, 50000, n)
        x = [randn(g, layers, n, h, d, dtype=dtype, scale=2.0) for h in (hq, max(hk, 1))]
        gy = [randn(g, *a.shape, dtype=dtype) for a in x]
        wt = [make_weight(g, kind, layers, a.shape[2], d, dtype) for a in x]
        nm = [fcg.Norm(a, 1e-5, offset) for a in wt]
        dx = [torch.full_like(a, float("nan")) for a in x]
        dw = [None if a is None else torch.full(nm[i].dweight_shape(layers, x[i].shape[2]), float("nan"), device="cuda")
              for i, a in enumerate(wt)]
        sides = 2 if hk else 1
        args = [a for i in range(sides) for a in (x[i], nm[i], gy[i], dx[i], dw[i])]
        fcg.fcg_norm_rope_backward(rope, dpos(pos), *args)
        torch.cuda.synchronize()
        first = [t.clone() for t in dx[:sides] + [t for t in dw[:sides] if t is not None]]
        for i in range(sides):
            check_grad(dx[i], dw[i], x[i], weights64(wt[i], offset, layers, x[i].shape[2], d), gy[i], 1e-5, pos, w, pairs, m,
                       dtype, f"{'qk'[i]} {kind}")
        fcg.fcg_norm_rope_backward(rope, dpos(pos), *args)        # the same bits again
        assert all(torch.equal(a, b) for a, b in zip(first, dx[:sides] + [t for t in dw[:sides] if t is not None]))


def test_gradient_in_place_of_either_input_and_one_side_turned_only():
    n, h, d = 100, 6, 128
    rope, w = make_rope(128, False)
    x, gy, weight = randn(gen(1), n, h, d), randn(gen(2), n, h, d), randn(gen(3), d)
    nm = fcg.Norm(weight)
    dx, dk, turned = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    fcg.fcg_norm_rope_backward(rope, dpos(range(n)), x, nm, gy, dx, None, None, None, gy, dk)
    fcg.fcg_rope_apply(rope, dpos(range(n)), gy, turned, flags=fcg.FCG_ROPE_BACKWARD)
    a, b = x.clone(), gy.clone()
    fcg.fcg_norm_rope_backward(rope, dpos(range(n)), a, nm, gy, a)
    fcg.fcg_norm_rope_backward(rope, dpos(range(n)), x, nm, b, b)
    torch.cuda.synchronize()
    check_grad(dx[None], None, x[None], weights64(weight, 0.0, 1, h, d), gy[None], 1e-6, range(n), w, False, 1.0, "bf16", "dx")
    assert torch.equal(bits(a), bits(dx)) and torch.equal(bits(b), bits(dx))
    assert torch.equal(bits(dk), bits(turned))


def test_gradient_of_no_tokens_clears_the_weights():
    rope, _ = make_rope(64, False)
    weight = torch.ones(3, 2, 64, device="cuda")
    x = torch.empty(3, 0, 2, 64, device="cuda")
    dw = torch.full((3, 2, 64), 7.0, device="cuda")
    fcg.fcg_norm_rope_backward(rope, dpos([]), x, fcg.Norm(weight), x, torch.empty_like(x), dw)
    assert not bool(dw.any())


def test_autograd_function():
    """The calls as forward and backward of an autograd function: the gradients autograd takes of the definition."""
    n, h, d, eps = 40, 4, 64, 1e-6
    rope, w = make_rope(64, True)
    pos = dpos(np.arange(100, 100 + n))

    class NormRope(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, weight):
            ctx.save_for_backward(x, weight)
            y = torch.empty_like(x)
            fcg.fcg_norm_rope_apply(rope, pos, x, fcg.Norm(weight, eps), y)
            return y

        @staticmethod
        def backward(ctx, gy):
            x, weight = ctx.saved_tensors
            dx, dw = torch.empty_like(x), torch.empty(1, h, d, device="cuda")
            fcg.fcg_norm_rope_backward(rope, pos, x, fcg.Norm(weight, eps), gy.contiguous(), dx, dw)
            return dx, dw[0]

    x = randn(gen(1), n, h, d, dtype="f32").requires_grad_()
    weight = randn(gen(2), h, d, dtype="f32").requires_grad_()
    gy = randn(gen(3), n, h, d, dtype="f32")
    NormRope.apply(x, weight).backward(gy)
    check_grad(x.grad[None], weight.grad[None], x.detach()[None], weights64(weight.detach(), 0.0, 1, h, d), gy[None], eps,
               np.arange(100, 100 + n), w, True, 1.0, "f32", "autograd")
    with pytest.raises(ValueError):
        fcg.fcg_norm_rope_apply(rope, pos, x, None, torch.empty_like(x))
    with pytest.raises(ValueError):
        fcg.fcg_norm_rope_apply(rope, pos, x.detach(), fcg.Norm(weight), torch.empty_like(x))


@pytest.mark.parametrize("dtype,hq,hkv,d", [("bf16", 32, 8, 128), ("bf16", 4, 2, 64), ("f32", 6, 3, 128)])
@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("own_form", [False, True])
def test_append_norm_stores_what_apply_gives(dtype, hq, hkv, d, page, own_form):
    """Runs of two sequences, holes, a large call whose plan is uploaded; the cache's own form and a handle's."""
    L, n_seq, T = 3, 70, 320
    rope, w = make_rope(d if own_form else d // 2, not own_form)
    for seq, pos in ((np.r_[np.zeros(20, int), np.ones(3, int)], np.r_[np.arange(5, 25), [300, 2, 3]]),
                     (np.arange(n_seq), np.arange(n_seq) * 4)):
        c = fcg.Cache(fcg.model_desc(L + 1, hq, hkv, d, 1e4, dtype), n_seq, T, page, 300 if page else 0)
        mem = cache_memory(c, dtype)
        for m in mem:
            m.fill_(7.0)
        n = len(seq)
        q, k, v = (randn(gen(i), L, n, h, d, dtype=dtype) for i, h in ((1, hq), (2, hkv), (3, hkv)))
        qw, kw = randn(gen(4), L, hq, d, dtype=dtype), randn(gen(5), d, dtype=dtype)
        qn, kn = fcg.Norm(qw, 1e-6, 1.0), fcg.Norm(kw, 1e-5)
        qo, qa, ka = torch.empty_like(q), torch.empty_like(q), torch.empty_like(k)
        fcg.fcg_append_norm(c, 1, seq, pos, k, v, kn, rope=None if own_form else rope, q=q, q_norm=qn, q_out=qo)
        fcg.fcg_norm_rope_apply(rope, dpos(pos), q, qn, qa, k, kn, ka)
        torch.cuda.synchronize()
        check_normed(qo, q, weights64(qw, 1.0, L, hq, d), 1e-6, pos, w, not own_form, 1.0, dtype, "q")
        if not own_form:
            assert torch.equal(bits(qo), bits(qa))
        for s in np.unique(seq):
            i = torch.as_tensor(np.flatnonzero(seq == s), device="cuda")
            K, V = (torch.stack([rows_of(c, m, l, s, pos[seq == s]) for l in range(1, L + 1)]) for m in mem)
            assert torch.equal(bits(V), bits(v[:, i]))
            if own_form:
                check_normed(K, k[:, i], weights64(kw, 0.0, L, hkv, d), 1e-5, pos[seq == s], w, False, 1.0, dtype, "keys")
            else:
                assert torch.equal(bits(K), bits(ka[:, i]))
            assert fcg.fcg_cache_export_layout(c, int(s), 1)[2].sum() == (seq == s).sum()
        assert bool((mem[0][0] == 7.0).all()) and fcg.fcg_cache_export_layout(c, 0, 0)[1] == 0
        c.close()


def test_calls_replay_in_a_graph_and_run_on_another_stream():
    n, hq, hk, d = 50, 8, 2, 128
    rope, w = make_rope(128, False)
    q, k, v = randn(gen(1), n, hq, d), randn(gen(2), n, hk, d), randn(gen(3), n, hk, d)
    gy, qw = randn(gen(4), n, hq, d), randn(gen(5), hq, d)
    nm, pos = fcg.Norm(qw), dpos(np.arange(n))
    qo, qo2, dx, dw = torch.empty_like(q), torch.empty_like(q), torch.empty_like(q), torch.empty(1, hq, d, device="cuda")
    ws = torch.empty(fcg.fcg_norm_rope_workspace(1, n, hq, 0, d), dtype=torch.uint8, device="cuda")
    c = fcg.Cache(fcg.model_desc(1, hq, hk, d, 1e4, "bf16"), 1, 64)
    seq, at = np.zeros(n, int), np.arange(n)

    def step():
        fcg.fcg_norm_rope_apply(rope, pos, q, nm, qo)
        fcg.fcg_append_norm(c, 0, seq, at, k, v, fcg.Norm(None), rope=rope, q=q, q_norm=nm, q_out=qo2, flags=fcg.FCG_REPLACE)
        fcg.fcg_norm_rope_backward(rope, pos, q, nm, gy, dx, dw, workspace=ws)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step()
    for seed in (11, 12, 13):
        q.copy_(randn(gen(seed), n, hq, d)), k.copy_(randn(gen(seed + 1), n, hk, d)), gy.copy_(randn(gen(seed + 2), n, hq, d))
        for t in (qo, qo2, dx, dw):
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (qo, qo2, dx, dw, rows_of(c, cache_memory(c, "bf16")[0], 0, 0, at))]
        step()
        torch.cuda.synchronize()
        want = (qo, qo2, dx, dw, rows_of(c, cache_memory(c, "bf16")[0], 0, 0, at))
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        check_normed(got[0][None], q[None], weights64(qw, 0.0, 1, hq, d), 1e-6, at, w, False, 1.0, "bf16", "replayed")
    with pytest.raises(ValueError):       # memory of the current stream's pool is not for another stream
        fcg.fcg_norm_rope_backward(rope, pos, q, nm, gy, dx, dw, stream=side)


def test_calls_larger_than_the_caches_equal_their_layers():
    """Rows past the last-level cache take nontemporal accesses; the same bits as one layer at a time."""
    n, hq, hk, d, L = 9000, 16, 4, 128, 6
    rope, _ = make_rope(128, False)
    q, k = randn(gen(1), L, n, hq, d), randn(gen(2), L, n, hk, d)
    nm = fcg.Norm(randn(gen(3), L, 1, d))
    pos = dpos(np.random.default_rng(1).integers(0, 9000, n))
    qo, ko, one = torch.empty_like(q), torch.empty_like(k), torch.empty_like(q[0])
    fcg.fcg_norm_rope_apply(rope, pos, q, nm, qo, k, nm, ko)
    for l in range(L):
        fcg.fcg_norm_rope_apply(rope, pos, q[l], fcg.Norm(nm.weight[l, 0]), one)
        assert torch.equal(bits(one), bits(qo[l]))


def test_a_norm_built_before_its_module_moves():
    """Weights made on the host, the norm with them, then moved to the GPU and replaced: each call takes the present ones."""
    d, hq, n = 64, 4, 33
    rope, w = make_rope(64, False)
    x, pos = randn(gen(1), 1, n, hq, d), np.arange(n)
    module = torch.nn.Module()
    module.weight = torch.nn.Parameter(torch.ones(d, dtype=torch.bfloat16), requires_grad=False)
    norm, y = fcg.Norm(module.weight), torch.empty_like(x)
    with pytest.raises(ValueError):
        fcg.fcg_norm_rope_apply(rope, dpos(pos), x, norm, y)
    module.cuda()
    for seed in (2, 3):
        fcg.fcg_norm_rope_apply(rope, dpos(pos), x, norm, y)
        torch.cuda.synchronize()
        check_normed(y, x, weights64(module.weight.data, 0.0, 1, hq, d), 1e-6, pos, w, False, 1.0, "bf16", f"weights {seed}")
        wide = randn(gen(seed), hq, 2 * d)
        module.weight.data = wide[:, d:] if seed == 2 else wide[0, :d].clone()
    fcg.fcg_norm_rope_apply(rope, dpos(pos), x, norm, y)
    dx, dw = torch.empty_like(x), torch.empty(norm.dweight_shape(1, hq), device="cuda")
    gy = randn(gen(5), 1, n, hq, d)
    fcg.fcg_norm_rope_backward(rope, dpos(pos), x, norm, gy, dx, dw)
    torch.cuda.synchronize()
    w64 = weights64(module.weight.data, 0.0, 1, hq, d)
    check_normed(y, x, w64, 1e-6, pos, w, False, 1.0, "bf16", "the last weights")
    check_grad(dx, dw, x, w64, gy, 1e-6, pos, w, False, 1.0, "bf16", "the last weights")


def test_a_step_of_no_tokens():
    c = fcg.Cache(fcg.model_desc(1, 4, 2, 64, 1e4, "bf16"), 1, 32, 16, 2)
    q, kv = (torch.empty(0, h, 64, dtype=torch.bfloat16, device="cuda") for h in (4, 2))
    norm = fcg.Norm(randn(gen(1), 64))
    fcg.fcg_append_norm(c, 0, [], [], kv, kv, norm, q=q, q_norm=norm, q_out=torch.empty_like(q))
    assert fcg.fcg_cache_export_layout(c, 0, 0)[1] == 0

"""Log probabilities, entropy, most likely tokens and the gradient of the logits on the GPU, against plain 64-bit forms."""
import math

import numpy as np
import pytest
import torch

from opsutil import DT, HALF_STEP, randn
from paper_2606_13097_amd import fcg

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")


@pytest.fixture(autouse=True)
def _gpu(request):
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    print(f"[gpu] {request.node.name}", flush=True)


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def bits(t):
    return t.contiguous().view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32)


def call(x, target=None, k=0, **kw):
    n = x.shape[0]
    out = {key: torch.full((n,), -77.0, device="cuda") for key in ("logprob", "entropy", "lse")}
    if target is None:
        out["logprob"] = None
    top = (torch.full((n, k), -77, dtype=torch.int32, device="cuda"), torch.full((n, k), -77.0, device="cuda")) if k else (None, None)
    fcg.fcg_token_logprobs(x, target, out["logprob"], out["entropy"], out["lse"], *top, **kw)
    torch.cuda.synchronize()
    return out, top


def top64(x, k):
    """Ids of the k largest of each row: larger first, lower id where equal, NaN last."""
    x = x.double().cpu().numpy()
    return np.stack([np.lexsort((np.arange(len(r)), np.where(np.isnan(r), 0.0, -r), np.isnan(r)))[:k] for r in x])


def check(x, target, out, top, what):
    """S adds at most V / 1024 + 32 terms in a row, each within 2^-22 (exp2) and 2^-24 of its exponent, whose mean under p
    is at most the entropy in bits (20 with a reference 2^40 off): S within rel = (V / 1024 + 90) 2^-24.  lse: that, and
    roundings of r + ln S; entropy: rel of log2 S and of U / S, each at most 60."""
    n, V = x.shape
    x64 = x.double()
    lse = torch.logsumexp(x64, -1)
    rel = (V / 1024 + 90) * 2.0 ** -24
    assert bool(((out["lse"].double() - lse).abs() <= rel + 2.0 ** -22 * lse.abs()).all()), f"{what}: lse"
    p = torch.softmax(x64, -1)
    ent = -torch.special.xlogy(p, p).sum(-1)
    assert bool(((out["entropy"].double() - ent).abs() <= 2 * 60 * rel).all()), f"{what}: entropy"
    rms = float((out["entropy"].double() - ent).square().mean().sqrt())     # roundings of either sign
    assert rms <= 6 * rel, f"{what}: entropy {rms:.2e}"
    if target is not None:
        ok = (target >= 0) & (target < V)
        xt = x64.gather(1, target.clamp(0, V - 1).long()[:, None])[:, 0]
        want = torch.where(ok, xt - lse, 0.0)
        tol = rel + 2.0 ** -23 * (want.abs() + (xt - x64.amax(-1)).abs() + 8)
        gone = torch.isinf(want)
        assert torch.equal(torch.isinf(out["logprob"]), gone), what
        assert bool(((out["logprob"].double() - want).abs() <= tol)[~gone].all()), f"{what}: logprob"
    if top[0] is not None:
        ids = torch.as_tensor(top64(x, top[0].shape[1]), device="cuda")
        assert torch.equal(top[0].long(), ids), f"{what}: ids"
        want = x64.gather(1, ids) - lse[:, None]
        gone = torch.isinf(want)
        assert torch.equal(torch.isinf(top[1]), gone), what
        tol = rel + 2.0 ** -23 * (want.abs() + 40)
        assert bool(((top[1].double() - want).abs() <= tol)[~gone].all()), f"{what}: top"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [1, 2, 7, 8, 9, 63, 64, 1000, 4096, 16384, 16391, 50021, 131072, 131075])
def test_rows_of_every_length(dtype, V):
    for n, k, pad, start in ((1, 20, 0, 0), (3, 64, 5, 1), (70, 1, 0, 3), (600, 5, 3, 0)):
        if n * V > 2e7:
            continue
        g = gen(V + n)
        flat = randn(g, start + n * (V + pad), dtype=dtype, scale=3.0)
        x = flat[start:].view(n, V + pad)[:, :V]
        target = torch.randint(-1, V + 2, (n,), generator=g, device="cuda", dtype=torch.int32)
        k = min(k, V)
        out, top = call(x, target, k)
        check(x, target, out, top, f"{dtype} {n} x {V}")
        none, _ = call(x, target, 0)
        assert all(torch.equal(none[key], out[key]) for key in none) or k
        check(x, target, none, (None, None), f"{dtype} {n} x {V}, no alternatives")
        again, top2 = call(x, target, k)
        assert all(torch.equal(again[key], out[key]) for key in out) and torch.equal(top[0], top2[0])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [2, 700])
def test_masked_rows(dtype, n):
    """Most tokens ruled out; fewer left than alternatives asked for; one left; a target that is ruled out."""
    V = 20000
    g = gen(n)
    x = randn(g, n, V, dtype=dtype)
    keep = torch.rand(n, V, generator=g, device="cuda") < 0.001
    keep[1] = False
    keep[1, 777] = True
    keep[:, 19999] |= torch.arange(n, device="cuda") % 2 == 0
    x = torch.where(keep, x, torch.full_like(x, -INF))
    target = torch.full((n,), 19999, dtype=torch.int32, device="cuda")
    out, top = call(x, target, 40)
    check(x, target, out, top, "masked")
    assert float(out["entropy"][1]) == 0.0 and float(out["lse"][1]) == float(x[1, 777])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [5, 40000])
def test_rows_that_leave_nothing_and_are_not_finite(dtype, V):
    low = torch.finfo(DT[dtype]).min
    x = randn(gen(V), 7, V, dtype=dtype)
    x[0] = -INF                       # nothing: no probability anywhere
    x[1] = low                        # the type's lowest value everywhere: uniform
    x[2] = -INF
    x[2, V // 2:] = low               # the same over a half
    x[3, 3] = NAN
    x[4, 1] = INF
    x[5, 1:] = low                    # one token against the lowest value
    x[6, V - 1] = -low                # and the highest
    target = torch.full((7,), 1, dtype=torch.int32, device="cuda")
    out, top = call(x, target, 4)
    assert float(out["lse"][0]) == -INF and float(out["logprob"][0]) == -INF and float(out["entropy"][0]) == 0.0
    assert top[0][0].tolist() == [0, 1, 2, 3] and bool((top[1][0] == -INF).all())
    for r, m in ((1, V), (2, V - V // 2)):
        assert abs(float(out["lse"][r]) - low) <= abs(low) * 2.0 ** -23
        assert abs(float(out["entropy"][r]) - math.log(m)) < 1e-4
    assert abs(float(out["logprob"][1]) + math.log(V)) < 1e-4 and float(out["logprob"][2]) == -INF
    assert top[0][1].tolist() == [0, 1, 2, 3] and top[0][2].tolist()[:2] == [V // 2, V // 2 + 1]
    assert all(math.isnan(float(out[key][3])) for key in out)
    assert top[0][3].tolist() == top64(x[3:4], 4)[0].tolist()
    assert float(out["lse"][4]) == INF and top[0][4, 0] == 1 and math.isnan(float(out["logprob"][4]))
    assert float(out["lse"][5]) == float(x[5, 0]) and float(out["entropy"][5]) == 0.0 and float(out["logprob"][5]) < -1e37
    assert float(out["lse"][6]) == -low and float(out["entropy"][6]) == 0.0
    all_nan = torch.full((1, V), NAN, dtype=DT[dtype], device="cuda")
    out, top = call(all_nan, None, 3)
    assert math.isnan(float(out["lse"])) and top[0].tolist() == [[0, 1, 2]]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 600])
def test_equal_and_ordered_logits(dtype, n):
    """Ties everywhere (the list of candidates overflows), ascending rows (every chunk has new ones), descending rows,
    all of the largest in the vectors of a few threads, signed zeros."""
    V = 33000
    i = torch.arange(V, device="cuda")
    rows = [torch.zeros(V, device="cuda"), (i % 3).float(), i / V * 20, -i / V * 20, (i // 8 % 512 < 5) * 4.0 + i / V,
            torch.where(i % 2 == 0, 0.0, -0.0) * 1.0, torch.where(i < 100, -5.0, 2.0), (i // 64 % 64 == 3) * (9.0 - i / V)]
    x = torch.stack(rows).to(DT[dtype])
    x = x.repeat(-(-n // len(rows)), 1)[:n] if n > 1 else x
    for k in (64, 7):
        for part in ([x] if n > 1 else [r[None] for r in x]):
            out, top = call(part, None, k)
            assert torch.equal(top[0].long(), torch.as_tensor(top64(part, k), device="cuda"))
            lse = torch.logsumexp(part.double(), -1)
            assert bool(((out["lse"].double() - lse).abs() <= (V / 1024 + 90) * 2.0 ** -24 + 2.0 ** -22 * lse.abs()).all())


@pytest.mark.parametrize("scale", [1e-3, 300.0, 3e4, 1e30])
def test_logits_of_every_size(scale):
    """Large logits cost no digits: their differences are formed from the values, not from rounded products."""
    x = randn(gen(3), 40, 30011, dtype="f32", scale=scale)
    x[:, 5] = x.amax(-1)               # a tie for the first place
    target = torch.full((40,), 5, dtype=torch.int32, device="cuda")
    out, top = call(x, target, 10)
    rest = torch.logsumexp(x.double() - x.double().amax(-1, keepdim=True), -1)     # (64 bits hold no ln 2 beside 1e30)
    lp = x.double()[:, 5] - x.double().amax(-1) - rest
    assert bool(((out["logprob"].double() - lp).abs() <= 150 * 2.0 ** -24 * (1 + lp.abs())).all())
    assert torch.equal(top[0].long(), torch.as_tensor(top64(x, 10), device="cuda"))
    p = torch.softmax(x.double(), -1)
    ent = -torch.special.xlogy(p, p).sum(-1)
    assert bool(((out["entropy"].double() - ent).abs() <= 120 * 60 * 2.0 ** -24).all())


def grad64(x, target, lse, ent, gl, gh, gs):
    x = x.double()
    lp = x - lse.double()[:, None]
    p = lp.exp()
    gl, gh, gs = (0.0 if g is None else g.double()[:, None] for g in (gl, gh, gs))
    e = 0.0 if ent is None else ent.double()[:, None]
    t = torch.full((len(x),), -1, device="cuda") if target is None else target.long()
    ok = ((t >= 0) & (t < x.shape[1]))[:, None]
    gl = torch.where(ok, torch.as_tensor(gl, dtype=torch.float64, device="cuda"), 0.0)
    dead = x == -INF
    lps = torch.where(dead, 0.0, lp)
    d = torch.where(dead, 0.0, p * (gs - gl - gh * (lps + e)))
    size = torch.where(dead, 0.0, p) * (abs(gs) + abs(gl) + abs(gh) * (abs(e) + lps.abs())) * (4 * lps.abs() + 16) * 2.0 ** -24
    hit = (torch.arange(x.shape[1], device="cuda") == t[:, None]) & ok
    return d + torch.where(hit, gl, 0.0), size + torch.where(hit, abs(gl) * 2.0 ** -23, 0.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [1, 7, 8, 9, 1000, 8192, 50021])
def test_gradient(dtype, V):
    """An exponent of -lp is off by 4 |lp| 2^-24 with its roundings and exp2 by 2^-22; sums of the row's factors round a
    few times: 16 more.  Every subset of the three gradients; strided rows that start anywhere; then in place."""
    for n, pad, start, which in ((1, 0, 0, 7), (33, 3, 1, 7), (5, 0, 0, 1), (5, 1, 3, 2), (5, 0, 0, 4), (3, 0, 0, 0)):
        g = gen(V + n)
        flat = randn(g, start + n * (V + pad), dtype=dtype, scale=3.0)
        x = flat[start:].view(n, V + pad)[:, :V]
        if V > 8:
            x[:, 3::5] = -INF
        target = torch.randint(-1, V + 1, (n,), generator=g, device="cuda", dtype=torch.int32)
        gl, gh, gs = (torch.randn(n, generator=g, device="cuda") if which >> i & 1 else None for i in range(3))
        out, _ = call(x, None)
        ent = out["entropy"] if which & 2 else None
        tg = target if which & 1 else None
        dflat = torch.full((1 + n * (V + 2),), 7.0, dtype=DT[dtype], device="cuda")
        dx = dflat[1:].view(n, V + 2)[:, :V]
        fcg.fcg_token_logprobs_backward(x, tg, out["lse"], ent, dx, g_logprob=gl, g_entropy=gh, g_lse=gs)
        torch.cuda.synchronize()
        ref, fp = grad64(x, tg, out["lse"], ent, gl, gh, gs)
        err = (dx.double() - ref).abs()
        assert bool((err <= HALF_STEP[dtype] * (ref.abs() + fp) + fp + 1e-37).all()), f"{dtype} {n} x {V} {which}"
        assert float(dflat[0]) == 7.0 and bool((dflat[1:].view(n, V + 2)[:, V:] == 7.0).all())
        keep = flat.clone()
        fcg.fcg_token_logprobs_backward(x, tg, out["lse"], ent, x, g_logprob=gl, g_entropy=gh, g_lse=gs)
        torch.cuda.synchronize()
        assert torch.equal(bits(x), bits(dx))
        if pad:
            assert torch.equal(bits(flat[start:].view(n, V + pad)[:, V:]), bits(keep[start:].view(n, V + pad)[:, V:]))


def test_gradient_of_rows_that_leave_nothing():
    x = torch.zeros(3, 500, device="cuda")
    x[0] = -INF
    x[1, 1:] = torch.finfo(torch.float32).min
    target = torch.tensor([5, 0, 9], dtype=torch.int32, device="cuda")
    one = torch.ones(3, device="cuda")
    out, _ = call(x, target)
    dx = torch.empty_like(x)
    fcg.fcg_token_logprobs_backward(x, target, out["lse"], out["entropy"], dx, g_logprob=one, g_entropy=one, g_lse=one)
    assert bool(torch.isfinite(dx).all()) and float(dx[0, 5]) == 1.0 and not bool(dx[0, :5].any())
    assert float(dx[1, 0]) == 1.0 and not bool(dx[1, 1:].any())


def test_autograd_function_against_torch_and_differences():
    V, n = 321, 6
    x = randn(gen(1), n, V, dtype="f32").requires_grad_()
    target = torch.randint(0, V, (n,), generator=gen(2), device="cuda", dtype=torch.int32)

    class Loss(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, target):
            lp, ent, lse = (torch.empty(n, device="cuda") for _ in range(3))
            fcg.fcg_token_logprobs(x, target, lp, ent, lse)
            ctx.save_for_backward(x, target, lse, ent)
            return lp, ent, lse

        @staticmethod
        def backward(ctx, gl, gh, gs):
            x, target, lse, ent = ctx.saved_tensors
            dx = torch.empty_like(x)
            fcg.fcg_token_logprobs_backward(x, target, lse, ent, dx, g_logprob=gl.contiguous(), g_entropy=gh.contiguous(),
                                            g_lse=gs.contiguous())
            return dx, None

    def loss(lp, ent, lse):
        return -lp.mean() - 0.1 * ent.sum() + 1e-2 * lse.square().sum()

    loss(*Loss.apply(x, target)).backward()
    y = x.detach().double().requires_grad_()
    lse = torch.logsumexp(y, -1)
    lp = y - lse[:, None]
    ref = loss(lp.gather(1, target.long()[:, None])[:, 0], -(lp.exp() * lp).sum(-1), lse)
    ref.backward()
    assert float((x.grad.double() - y.grad).abs().max()) < 2e-6
    h = 1e-6
    for r, c in ((0, 0), (1, int(target[1])), (5, 320)):
        vals = []
        for s in (h, -h):
            z = x.detach().double().clone()
            z[r, c] += s
            lse = torch.logsumexp(z, -1)
            lp = z - lse[:, None]
            vals.append(float(loss(lp.gather(1, target.long()[:, None])[:, 0], -(lp.exp() * lp).sum(-1), lse)))
        assert abs((vals[0] - vals[1]) / (2 * h) - float(x.grad[r, c])) < 1e-5
    with pytest.raises(ValueError):
        fcg.fcg_token_logprobs(x, target, torch.empty(n, device="cuda"))


def test_replays_in_a_graph_on_another_stream():
    n, V, k = 5, 70001, 8
    x = randn(gen(1), n, V)
    target = torch.randint(0, V, (n,), generator=gen(2), device="cuda", dtype=torch.int32)
    lp, ent, lse = (torch.empty(n, device="cuda") for _ in range(3))
    ids, tlp, dx = torch.empty(n, k, dtype=torch.int32, device="cuda"), torch.empty(n, k, device="cuda"), torch.empty_like(x)
    ws = torch.empty(fcg.fcg_token_logprobs_workspace(n, V, k), dtype=torch.uint8, device="cuda")
    g = torch.ones(n, device="cuda")

    def step():
        fcg.fcg_token_logprobs(x, target, lp, ent, lse, ids, tlp, workspace=ws)
        fcg.fcg_token_logprobs_backward(x, target, lse, ent, dx, g_logprob=g, g_entropy=g)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step()
    for seed in (1, 2, 3):
        x.copy_(randn(gen(seed), n, V))
        for t in (lp, ent, lse, tlp, dx):
            t.fill_(NAN)
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (lp, ent, lse, ids, tlp, dx)]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (lp, ent, lse, ids, tlp, dx)))
        check(x, target, dict(logprob=got[0], entropy=got[1], lse=got[2]), (got[3], got[4]), "replayed")
    with pytest.raises(ValueError):
        fcg.fcg_token_logprobs(x, target, lp, stream=side)


def test_offsets_past_32_bits():
    """Rows further apart than 2^31 bytes and a tensor of more than 2^32."""
    n, V, step = 3, 1000, 1 << 30
    flat = torch.empty((n - 1) * step + V, dtype=torch.bfloat16, device="cuda")
    x = torch.as_strided(flat, (n, V), (step, 1))
    x.copy_(randn(gen(1), n, V))
    target = torch.tensor([1, 2, 3], dtype=torch.int32, device="cuda")
    out, top = call(x, target, 5)
    check(x, target, out, top, "far rows")
    g = torch.ones(n, device="cuda")
    ref, dx = torch.empty(n, V, dtype=torch.bfloat16, device="cuda"), torch.empty(n, V, dtype=torch.bfloat16, device="cuda")
    fcg.fcg_token_logprobs_backward(x.contiguous(), target, out["lse"], None, ref, g_logprob=g)
    fcg.fcg_token_logprobs_backward(x, target, out["lse"], None, dx, g_logprob=g)
    assert torch.equal(dx, ref)
    many = torch.empty(40001, 60000, dtype=torch.bfloat16, device="cuda")
    many[-1] = randn(gen(2), 60000)
    many[:-1] = 0
    out, _ = call(many)
    assert abs(float(out["lse"][-1]) - float(torch.logsumexp(many[-1].double(), 0))) < 1e-4
    assert bool(((out["lse"][:-1] - math.log(60000)).abs() < 1e-4).all())


def test_perplexities_reach_the_locality_score():
    """Retrieved functions' tokens to what stays in device memory: log probabilities, perplexities, the update step."""
    lengths = [30, 7, 120, 1]
    V, n = 5000, sum(lengths)
    x = randn(gen(1), n, V, scale=2.0)
    x[30:37, 11] += 20.0                     # a function that the model predicts well
    target = torch.full((n,), 11, dtype=torch.int32, device="cuda")
    lp = torch.empty(n, device="cuda")
    fcg.fcg_token_logprobs(x, target, lp)
    loc = fcg.Locality(4, alpha=0.0, beta=0.0, gamma=1.0)
    fcg.fcg_locality_measure_ppl(loc, [2, 0, 3, 1], lengths, lp)
    want = np.exp([-float(p.double().mean()) for p in torch.split(lp, lengths)])[[1, 3, 0, 2]]
    np.testing.assert_allclose(fcg.fcg_locality_scores(loc), want / want.max(), rtol=1e-12)
    desc = fcg.model_desc(1, 4, 2, 64, 1e4, "bf16")
    lib = fcg.Library(desc, 64, 4)
    for _ in range(4):
        k = randn(gen(3), 1, 16, 2, 64)
        fcg.fcg_lib_add_segment(lib, 16, 0, k, k)
    fcg.fcg_lib_host_reserve(lib, 64)
    fcg.fcg_lib_update_residency(lib, loc, 3 * 16 * 2 * 2 * 64 * 2)
    torch.cuda.synchronize()
    assert [fcg.fcg_lib_segment_state(lib, s)[0] for s in range(4)] == [s != int(np.argmin(want)) for s in range(4)]
    before = fcg.fcg_locality_scores(loc)
    lp[3] = -INF
    with pytest.raises(fcg.FcgError):
        fcg.fcg_locality_measure_ppl(loc, [0, 1], [2, 2], lp)
    assert np.array_equal(before, fcg.fcg_locality_scores(loc))


def test_perplexities_are_not_measured_while_capturing():
    loc = fcg.Locality(2)
    lp, x = torch.zeros(2, device="cuda"), torch.zeros(1, device="cuda")
    status, graph = fcg.FCG_OK, torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        try:
            fcg.fcg_locality_measure_ppl(loc, [0], [2], lp)
        except fcg.FcgError as e:
            status = e.status
        x += 1.0
    assert status == fcg.FCG_ESTATE
    for n in range(1, 4):                    # the capture went on
        graph.replay()
        torch.cuda.synchronize()
        assert float(x) == n
    fcg.fcg_locality_measure_ppl(loc, [0], [2], lp)

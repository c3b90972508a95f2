"""Log probabilities and entropies of confident rows: one token far above the others, against the 64-bit definition."""
import math

import pytest
import torch

from opsutil import DT, randn
from paper_2606_13097_amd import fcg

pytestmark = pytest.mark.gpu


def call(x, target, k):
    n = x.shape[0]
    lp, ent, lse, tlp = (torch.full(s, -77.0, device="cuda") for s in ((n,), (n,), (n,), (n, max(k, 1))))
    ids = torch.full((n, max(k, 1)), -77, dtype=torch.int32, device="cuda")
    fcg.fcg_token_logprobs(x, target, lp, ent, lse, *((ids, tlp) if k else ()))
    torch.cuda.synchronize()
    return lp, ent, lse, ids, tlp


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [32000, 131072, 131075])
@pytest.mark.parametrize("n,k", [(1, 20), (64, 0), (64, 20), (1100, 0)])
def test_confident_rows_keep_their_digits(dtype, V, n, k):
    """Peaks of 20 to 45 in rows of spread 2.5, wherever they stand.  With the sum taken about the row's maximum M it is
    1 + T, T the mass of the others.  Added to the peak, a sum e of others is off by at most min(2^-24 (1 + T), e), in
    V / 4096 + 40 additions (of a vector's sum to an accumulator, 512 or more of these; lanes, waves, splits): by
    min(2 T, (V / 2048 + 40) 2^-24 (1 + T)) in all.  A term of T is off by 2.5 |x - M| 2^-24 (difference, product,
    constant) and 2^-22 (the exponential) of itself, as is its part of U = sum e^(x - M) (x - M), which V / 256 + 60
    additions of one sign round to 2^-24 of it.  ln S and U / S: 4 more roundings.  Logarithms of S >= 1 are not
    negative and neither is -U, so no log probability is above 0 and no entropy below."""
    print(f"[gpu] confident rows {dtype} {n} x {V}, {k} alternatives", flush=True)
    g = torch.Generator(device="cuda").manual_seed(V + n)
    x = randn(g, n, V, dtype=dtype, scale=2.5)
    at = torch.randint(0, V, (n,), generator=g, device="cuda")
    at[0] = V - 1
    peaks = torch.tensor([20.0, 25.0, 27.0, 30.0, 33.0, 35.0, 45.0], device="cuda")
    x[torch.arange(n, device="cuda"), at] = peaks[torch.arange(n, device="cuda") % 7].to(DT[dtype])
    lp, ent, lse, ids, tlp = call(x, at.int(), k)
    for r0 in range(0, n, 100):
        s = slice(r0, r0 + 100)
        d = x[s].double()
        M = d.gather(1, at[s, None])
        assert bool((d.amax(-1, keepdim=True) == M).all())
        d = d - M
        e = d.exp()
        far = float(-d.min())
        d.scatter_(1, at[s, None], 0.0)
        e.scatter_(1, at[s, None], 0.0)
        T, U = e.sum(-1), (e * d).sum(-1)
        ln_s = torch.log1p(T)
        H = ln_s - U / (1 + T)
        u = 2.0 ** -24
        off = torch.minimum(2 * T, (V / 2048 + 40) * u * (1 + T)) + (2.5 * far + 8) * u * T
        assert bool((lp[s] <= 0).all()) and bool((ent[s] >= 0).all())
        err = (lp[s].double() + ln_s).abs()
        assert bool((err <= off + 4 * u * ln_s).all()), f"log probability {float((err - off).max()):.2e} past the bound"
        err = (ent[s].double() - H).abs()
        tol = off + (V / 256 + 2.5 * far + 70) * u * U.abs() + 4 * u * H
        assert bool((err <= tol).all()), f"entropy {float((err - tol).max()):.2e} past the bound"
        assert bool(((lse[s].double() - M[:, 0] - ln_s).abs() <= off + 4 * u * ln_s + u * M[:, 0].abs() * 2).all())
        if k:
            assert torch.equal(ids[s, 0].long(), at[s]) and torch.equal(tlp[s, 0], lp[s])


@pytest.mark.parametrize("n", [2, 1100])
def test_two_tokens_share_a_row(n):
    """Two tokens far above the others, from equal to a step apart that the sum's reference does not follow: entropy of
    two, within 16 roundings of sums near 1 (and 2^-22 for each exponential)."""
    print(f"[gpu] two tokens, {n} rows", flush=True)
    V = 50021
    g = torch.Generator(device="cuda").manual_seed(n)
    x = randn(g, n, V, dtype="f32")
    gap = torch.linspace(0, 4, n, device="cuda")
    x[:, 77], x[:, 40000] = 60.0, 60.0 - gap
    x[1::2, 40000], x[1::2, 77] = 60.0, 60.0 - gap[1::2]
    target = torch.full((n,), 77, dtype=torch.int32, device="cuda")
    lp, ent, *_ = call(x, target, 0)
    d = (x[:, [77, 40000]].double() - x[:, [77, 40000]].double().amax(-1, keepdim=True))
    ref = torch.log_softmax(d, -1)
    H = -(ref.exp() * ref).sum(-1)
    assert bool(((lp.double() - ref[:, 0]).abs() <= 24 * 2.0 ** -24 * (1 + ref[:, 0].abs())).all())
    assert bool(((ent.double() - H).abs() <= 48 * 2.0 ** -24).all()) and bool((lp <= 0).all())
    assert math.isclose(float(ent[0]), math.log(2), rel_tol=1e-6)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,V", [(1, 5), (3, 4099), (2, 131075), (1100, 20011)])
def test_alternatives_change_no_statistics(dtype, n, V):
    """A call with alternatives reads a row in other pieces: sums of V / 1024 + 32 terms in another order, each within
    2^-22 and 3 roundings of differences of at most 64, so ln S within (V / 1024 + 90) 2^-24 of the 64-bit one (the entropy 64
    times that) on both sides, and roundings of the results."""
    print(f"[gpu] with and without alternatives {dtype} {n} x {V}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(V)
    x = randn(g, n, V, dtype=dtype, scale=3.0)
    target = torch.randint(0, V, (n,), generator=g, device="cuda", dtype=torch.int32)
    a, b = call(x, target, 0), call(x, target, min(20, V))
    rel = 2 * (V / 1024 + 90) * 2.0 ** -24
    for i, (p, q) in enumerate(zip(a[:3], b[:3])):
        assert bool(((p.double() - q.double()).abs() <= rel * (64 if i == 1 else 1) + 2.0 ** -22 * p.abs()).all())

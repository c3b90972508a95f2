"""Plain 64-bit forms of row norms with a rotary turn, and bounds that count the roundings of the kernels."""
import torch

from opsutil import HALF_STEP, turn64

EPS24 = 2.0 ** -24


def weights64(w, offset, layers, heads, d):
    """Norm weights with their offset as float64 [layers][1][heads][d]; w: as fcg.Norm takes it, or None."""
    if w is None:
        return torch.ones((), dtype=torch.float64)
    w = w.double() + offset
    while w.dim() < 3:
        w = w[None]
    return w.expand(layers, heads, d)[:, None]


def norm64(x, w, eps):
    """x [layers][n][heads][d] float64 (w of weights64) normalised."""
    return x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * w


def pair_size(x, rot, pairs):
    """|a| + |b| of each element's rotary pair; |x| where nothing turns."""
    a = x.abs().clone()
    ia, ib = (slice(0, rot, 2), slice(1, rot, 2)) if pairs else (slice(0, rot // 2), slice(rot // 2, rot))
    both = a[..., ia] + a[..., ib]
    a[..., ia] = both
    a[..., ib] = both
    return a


def check_normed(got, x, w, eps, pos, freqs, pairs, m, dtype, what):
    """One rounding to dtype after fp32 work.  The sum of 64 or 128 squares passes at most 16 + 4 additions and 16
    products (36 half steps of 2^-24, all terms positive), the mean, eps, root and quotient 8 more; the root halves what
    comes before it, so the scale is within 26 of them; times weight, offset and value 4.  The turn: cos and sin (with
    the factor) within 2^-22, 4 half steps, products and sum 3, of |a| + |b|.  37 in all; 40 counted."""
    n = norm64(x.double(), w.to(x.device), eps)
    ref = turn64(n, pos, freqs, pairs, m)
    fp = 40 * EPS24 * max(m, 1.0) * pair_size(n, 2 * len(freqs), pairs)
    tol = HALF_STEP[dtype] * (ref.abs() + fp) + fp + 1e-37
    err = (got.double() - ref).abs()
    assert bool((err <= tol).all()), f"{what}: {float((err - tol).max()):.3e} past the bound"


def grad64(x, w, gy, eps, pos, freqs, pairs, m):
    """-> (dx, dw before it is summed over rows and shared heads) by autograd of the 64-bit definition."""
    x = x.detach().double().clone().requires_grad_()
    full = (w.to(x.device) + torch.zeros_like(x)).detach().requires_grad_()
    with torch.enable_grad():
        turn64_grad = turn64(gy.double(), pos, freqs, pairs, m, sign=-1.0)   # the transposed turn
        return torch.autograd.grad(norm64(x, full, eps), (x, full), turn64_grad)


def check_grad(got_dx, got_dw, x, w, gy, eps, pos, freqs, pairs, m, dtype, what):
    """dx: the turned gradient is within 7 half steps of its pair's size, the scale within 26 (check_normed), products
    with weights and scale 4, the mean of d products within 40 of the mean of their sizes, then 4 more: each term of
    s (g - xhat mean(g xhat)) is within 100 half steps of its size.  dw: a term within 40, and the sum over N rows
    adds at most N + 64 roundings of the sum of sizes."""
    dx, dwr = grad64(x, w, gy, eps, pos, freqs, pairs, m)
    x64, g64 = x.double(), gy.double()
    s = 1 / torch.sqrt((x64 * x64).mean(-1, keepdim=True) + eps)
    size = pair_size(g64, 2 * len(freqs), pairs) * max(m, 1.0)
    xh = (x64 * s).abs()
    gw = size * w.to(x.device).abs()
    fp = 100 * EPS24 * s * (gw + xh * (gw * xh).mean(-1, keepdim=True))
    tol = HALF_STEP[dtype] * (dx.abs() + fp) + fp + 1e-37
    err = (got_dx.double() - dx).abs()
    assert bool((err <= tol).all()), f"{what}: dx {float((err - tol).max()):.3e} past the bound"
    if got_dw is None:
        return
    L, n, H, d = x.shape
    per_head = got_dw.shape[1] > 1
    over = 1 if per_head else (1, 2)
    ref = dwr.sum(over).view(got_dw.shape)
    rows = n * (1 if per_head else H)
    tol = (rows + 104) * EPS24 * (size * xh).sum(over).view(got_dw.shape) + 1e-37
    err = (got_dw.double() - ref).abs()
    assert bool((err <= tol).all()), f"{what}: dw {float((err - tol).max()):.3e} past the bound"

"""Bounds of prefix attention that count the roundings its kernels make, and no others.

bf16 caches: scores and sums are fp32; the probabilities are rounded to bf16 (the matrix product takes both its operands
in one type), split partials to fp16 with a power of two a row, the result to bf16."""
import torch

from opsutil import HALF_STEP

# Relative Frobenius error.  A rounding to bf16 is off by up to 2^-8 of the power of two below a value, evenly spread: an
# rms of 2^-8 / sqrt(3) of that power.  Against values whose logarithms are spread evenly (mean square 3 / (2 ln 2) of it)
# that is 1.53e-3, against normal ones 1.66e-3.  The probabilities and the result make two such roundings, independent of
# each other: 2.2e-3 to 2.35e-3; fp16 partials add an eighth of one, 0.2e-3, in square.  bf16 partials would make
# three, 2.65e-3 to 2.9e-3.
NORM_LIMIT = 2.5e-3


def check_attend_tight(got, got_lse, ref, dtype, n_keys, d, what, spread=False):
    """got against (out, lse, mass, reach) of attend64.  fp32: d products and sums of a score off by (d + 8) 2^-24 of
    sum |q k|, each probability by that share (delta), sums over the keys by n 2^-24.  bf16 rounds each probability by
    2^-8 and each partial by 2^-11 of its share of sum p |v|, and the result by 2^-8 of itself.  spread: many keys of like
    weight, so that the norm bound holds too."""
    out, lse, mass, reach = ref
    delta = (d + 8) * 2.0 ** -24 * reach + (n_keys + 32) * 2.0 ** -24
    tol = HALF_STEP[dtype] * out.abs() + 2.1 * delta[..., None] * mass + 1e-30
    if dtype == "bf16":
        tol = tol + (1 + 2.0 ** -3) * 2.0 ** -8 * 1.01 * mass
    assert not torch.isnan(got.float()).any(), what
    err = got.double() - out
    assert bool((err.abs() <= tol).all()), f"{what}: {float((err.abs() - tol).max()):.3e} past the bound"
    if spread and dtype == "bf16":
        rel = float(err.norm() / out.norm())
        assert rel <= NORM_LIMIT, f"{what}: relative norm {rel:.3e}"
    if got_lse is not None:
        empty = torch.isinf(lse)
        assert torch.equal(torch.isinf(got_lse) & (got_lse < 0), empty), what
        e = (got_lse.double() - lse).abs()[~empty]
        assert bool((e <= (delta + 2.0 ** -21 * (1 + lse.abs()))[~empty]).all()), f"{what}: lse"

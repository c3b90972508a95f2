"""Plain 64-bit forms of the rotary, append and prefix-attention calls, and error bounds for them.

Bounds count roundings: a result rounded to bf16 is off by at most 2^-8 of its value (half a step of 8
significant bits), to fp32 by 2^-24."""
import ctypes
import math

import numpy as np
import torch

from paper_2606_13097_amd import fcg

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def freqs64(rot, theta, kind="plain", factor=1.0, orig=0.0, lo=1.0, hi=32.0):
    if kind == "ntk":
        theta = theta * factor ** (rot / (rot - 2))
    w = theta ** (-2.0 * np.arange(rot // 2) / rot)
    if kind == "linear":
        w = w / factor
    if kind == "parts":
        c = np.clip((orig * w / (2 * math.pi) - lo) / (hi - lo), 0.0, 1.0)
        w = w * ((1 - c) / factor + c)
    return w


def turn64(x, pos, w, pairs, m=1.0, sign=1.0):
    """x [..., n, heads, d] (any float type) turned at pos [n], in float64 on x's device."""
    x = x.to(torch.float64)
    a = torch.as_tensor(np.asarray(pos, dtype=np.float64), device=x.device)[:, None] * torch.as_tensor(w, device=x.device)
    c, s = (m * a.cos())[:, None, :], (sign * m * a.sin())[:, None, :]
    r = 2 * len(w)
    y = x.clone()
    ia, ib = (slice(0, r, 2), slice(1, r, 2)) if pairs else (slice(0, r // 2), slice(r // 2, r))
    y[..., ia] = x[..., ia] * c - x[..., ib] * s
    y[..., ib] = x[..., ib] * c + x[..., ia] * s
    return y


def check_turned(got, ref, x, w, pairs, m, dtype, what):
    """One rounding to dtype, after an fp32 turn: cos and sin (with the factor) are within 2^-22 of theirs
    and the two products and the sum round by 2^-24 each, all relative to |a| + |b| of the pair; dimensions
    past the turned ones are copied bit for bit."""
    r = 2 * len(w)
    assert torch.isfinite(got.float()).all(), what
    assert torch.equal(got[..., r:], x[..., r:]), f"{what}: unturned dimensions"
    ia, ib = (slice(0, r, 2), slice(1, r, 2)) if pairs else (slice(0, r // 2), slice(r // 2, r))
    size = x[..., ia].double().abs() + x[..., ib].double().abs()
    both = torch.empty_like(ref[..., :r])
    both[..., ia] = size
    both[..., ib] = size
    tol = HALF_STEP[dtype] * ref[..., :r].abs() + (2.0 ** -22 + 3 * 2.0 ** -24) * max(m, 1.0) * both * 1.01
    err = (got[..., :r].double() - ref[..., :r]).abs()
    assert bool((err <= tol).all()), f"{what}: {float((err - tol).max()):.3e} past the bound"


def attend64(q, K, V, pos, prefix_len):
    """q [n][hq][d]; K, V [T][hkv][d] of one sequence (prefix and own joined by position); row t sees keys
    0 .. pos[t].  -> out, lse, sum p |v|, max over keys of sum |q k| / sqrt(d)."""
    n, hq, d = q.shape
    T, hkv, _ = K.shape
    g = hq // hkv
    q, K, V = q.double(), K.double(), V.double()
    out, lse, mass, reach = (torch.zeros(s, dtype=torch.float64, device=q.device) for s in ((n, hq, d), (n, hq), (n, hq, d), (n, hq)))
    lse.fill_(-math.inf)
    for t in range(n):
        if pos[t] < 0:
            continue
        k, v = K[:pos[t] + 1], V[:pos[t] + 1]
        for h in range(hkv):
            z = q[t, h * g:(h + 1) * g] @ k[:, h].T / math.sqrt(d)
            p = torch.softmax(z, -1)
            sl = slice(h * g, (h + 1) * g)
            out[t, sl], mass[t, sl] = p @ v[:, h], p @ v[:, h].abs()
            lse[t, sl] = torch.logsumexp(z, -1)
            reach[t, sl] = (q[t, sl].abs() @ k[:, h].abs().T / math.sqrt(d)).amax(-1)
    return out, lse, mass, reach


def check_attend(got, got_lse, ref, dtype, n_keys, d, what):
    """fp32 scores: d products and sums off by (d + 8) 2^-24 of sum |q k|, so each probability by that share
    (delta); sums over the keys add n 2^-24.  bf16 also rounds the probabilities, the partial outputs and the
    result by 2^-8 each; the first two act on sum p |v|."""
    out, lse, mass, reach = ref
    assert not torch.isnan(got.float()).any(), what
    delta = (d + 8) * 2.0 ** -24 * reach + (n_keys + 32) * 2.0 ** -24
    tol = HALF_STEP[dtype] * out.abs() + 2.1 * delta[..., None] * mass + 1e-30
    if dtype == "bf16":
        tol = tol + 2.02 * 2.0 ** -8 * mass
    err = (got.double() - out).abs()
    assert bool((err <= tol).all()), f"{what}: {float((err - tol).max()):.3e} past the bound"
    if got_lse is not None:
        empty = torch.isinf(lse)
        assert torch.equal(torch.isinf(got_lse) & (got_lse < 0), empty), what
        e = (got_lse.double() - lse).abs()[~empty]
        assert bool((e <= (delta + 2.0 ** -21 * (1 + lse.abs()))[~empty]).all()), f"{what}: lse"


class _Memory:
    def __init__(self, ptr, n, es, keep):
        self.keep = keep
        self.__cuda_array_interface__ = {"shape": (n,), "typestr": "<f4" if es == 4 else "<i2", "data": (ptr, False),
                                         "version": 2}


def cache_memory(cache, dtype):
    """K and V of all layers as tensors that share the cache's memory."""
    d = cache.desc
    shape = (d.n_layers, cache.n_pages, d.n_kv_heads, 16, d.head_dim) if cache.page_size else \
        (d.n_layers, cache.n_seqs, d.n_kv_heads, cache.max_tokens, d.head_dim)
    es = 4 if dtype == "f32" else 2
    out = []
    for ptr in fcg.fcg_cache_device_ptrs(cache, 0):
        m = torch.as_tensor(_Memory(ptr, math.prod(shape), es, cache), device="cuda")
        out.append((m if es == 4 else m.view(torch.bfloat16)).view(shape))
    return out


def rows_of(cache, mem, layer, seq, positions):
    """Rows [n][hkv][d] of a cache's memory tensor at positions of a sequence."""
    positions = torch.as_tensor(np.asarray(positions, dtype=np.int64))
    if not cache.page_size:
        return mem[layer, seq][:, positions].transpose(0, 1)
    pt, _, _ = fcg.fcg_cache_export_layout(cache, seq, layer)
    pages = torch.as_tensor(pt.astype(np.int64))[positions // 16]
    assert bool((pages >= 0).all())
    return mem[layer][pages, :, positions % 16]


def randn(g, *shape, dtype="bf16", scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(DT[dtype])

"""Rotary forms, append, graft in a rotary form and prefix attention on the GPU, against plain 64-bit forms."""
import math

import numpy as np
import pytest
import torch

from opsutil import (DT, HALF_STEP, attend64, cache_memory, check_attend, check_turned, freqs64, randn, rows_of, turn64)
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
    return t.view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32)


KINDS = {"plain": 0, "linear": 1, "ntk": 2, "parts": 3}


def make_rope(rot, pairs=False, kind="plain", theta=1e4, m=1.0):
    w = freqs64(rot, theta, kind, 4.0, 32768.0)
    return fcg.fcg_rope_create(rot, theta, layout=int(pairs), scaling=KINDS[kind], factor=4.0, orig_tokens=32768,
                               attn_factor=m), w


# ------------------------------------------------------------------ rope

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("d,rot", [(128, 128), (128, 112), (128, 32), (64, 64), (64, 16), (64, 48)])
def test_rope_apply_all_forms(dtype, pairs, d, rot):
    for kind, m, n, layers, hq, hk, top in (("plain", 1.0, 1, 1, 4, 1, 3), ("parts", 1.25, 77, 3, 5, 2, 200000),
                                             ("ntk", 0.5, 300, 1, 1, 0, 5000), ("linear", 1.0, 1500, 2, 8, 8, 4000)):
        g = gen(rot + n)
        rope, w = make_rope(rot, pairs, kind, m=m)
        pos = np.random.default_rng(n).integers(-top, top, n, endpoint=True)
        q, k = randn(g, layers, n, hq, d, dtype=dtype), randn(g, layers, n, hk, d, dtype=dtype)
        qo, ko = torch.empty_like(q), torch.empty_like(k)
        dpos = torch.as_tensor(pos, dtype=torch.int32, device="cuda")
        for flags, sign in ((0, 1.0), (fcg.FCG_ROPE_BACKWARD, -1.0)):
            qo.fill_(float("nan")), ko.fill_(float("nan"))
            fcg.fcg_rope_apply(rope, dpos, q, qo, k if hk else None, ko if hk else None, flags=flags)
            torch.cuda.synchronize()
            for x, y, name in ((q, qo, "q"), (k, ko, "k")):
                if x.numel():
                    check_turned(y, turn64(x, pos, w, pairs, m, sign), x, w, pairs, m, dtype, f"{name} {kind} {sign}")


@pytest.mark.parametrize("dtype,layers", [("bf16", 11), ("f32", 11), ("bf16", 23)])
def test_rope_apply_of_many_layers_in_place(dtype, layers):
    """Blocks that take several layers, not all as many; every layer from other rows, input and output the same."""
    n, hq, hk, d = 700, 8, 4, 128
    rope, w = make_rope(96, True, m=1.5)
    pos = np.random.default_rng(layers).integers(0, 30000, n)
    x = randn(gen(layers), layers, n, hq + hk + 1, d, dtype=dtype)
    was = x.clone()
    fcg.fcg_rope_apply(rope, torch.as_tensor(pos, dtype=torch.int32, device="cuda"), x[:, :, :hq], x[:, :, :hq],
                       x[:, :, hq:hq + hk], x[:, :, hq:hq + hk])
    torch.cuda.synchronize()
    ref = turn64(was[:, :, :hq + hk], pos, w, True, 1.5)
    check_turned(x[:, :, :hq + hk], ref, was[:, :, :hq + hk], w, True, 1.5, dtype, "in place")
    assert torch.equal(bits(x[:, :, hq + hk:].contiguous()), bits(was[:, :, hq + hk:].contiguous()))


@pytest.mark.parametrize("page", [0, 16])
def test_append_of_many_layers(page):
    """The same appending: pages, caches and q_out of every layer."""
    L, n, hq, hkv, d = 13, 300, 16, 4, 128
    rope, w = make_rope(64)
    c = fcg.Cache(fcg.model_desc(L + 2, hq, hkv, d, 1e4, "bf16"), 2, 400, page, 60 if page else 0)
    mem = fill_memory(c, "bf16", 7.0)
    seq, pos = np.r_[np.zeros(200, int), np.ones(100, int)], np.r_[np.arange(3, 203), np.arange(50, 150)]
    q, k, v = randn(gen(1), L, n, hq, d), randn(gen(2), L, n, hkv, d), randn(gen(3), L, n, hkv, d)
    qo = torch.empty_like(q)
    fcg.fcg_append(c, 1, seq, pos, k, v, rope=rope, q=q, q_out=qo, n_layers=L)
    torch.cuda.synchronize()
    check_turned(qo, turn64(q, pos, w, False), q, w, False, 1.0, "bf16", "q")
    for s in (0, 1):
        i = torch.as_tensor(np.flatnonzero(seq == s), device="cuda")
        K, V = (torch.stack([rows_of(c, m, l, s, pos[seq == s]) for l in range(1, L + 1)]) for m in mem)
        check_turned(K, turn64(k[:, i], pos[seq == s], w, False), k[:, i], w, False, 1.0, "bf16", f"keys of {s}")
        assert torch.equal(bits(V.contiguous()), bits(v[:, i].contiguous()))
    for m in mem:
        assert bool((m[0] == 7.0).all()) and bool((m[L + 1] == 7.0).all())
    c.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("offset", [0, 1, 3])
def test_rope_apply_takes_slices_any_start_and_in_place(dtype, offset):
    """q and k as slices of a fused projection that starts at any element; written in place and next to it."""
    n, hq, hk, d = 37, 6, 2, 64
    rope, w = make_rope(48, True, m=1.5)
    flat = randn(gen(offset), offset + n * (hq + 2 * hk) * d + 5, dtype=dtype)
    x = flat[offset:offset + n * (hq + 2 * hk) * d].view(n, hq + 2 * hk, d)
    keep = flat.clone()
    pos = np.arange(1000, 1000 + n)
    dpos = torch.as_tensor(pos, dtype=torch.int32, device="cuda")
    out = torch.full((n, hk + hq, d + 0), float("nan"), dtype=DT[dtype], device="cuda")
    fcg.fcg_rope_apply(rope, dpos, x[:, :hq], out[:, hk:], x[:, hq:hq + hk], out[:, :hk])
    torch.cuda.synchronize()
    assert torch.equal(bits(flat), bits(keep))
    q0, k0 = x[:, :hq].clone(), x[:, hq:hq + hk].clone()
    check_turned(out[:, hk:], turn64(q0, pos, w, True, 1.5), q0, w, True, 1.5, dtype, "q slice")
    check_turned(out[:, :hk], turn64(k0, pos, w, True, 1.5), k0, w, True, 1.5, dtype, "k slice")
    fcg.fcg_rope_apply(rope, dpos, x[:, :hq], x[:, :hq], x[:, hq:hq + hk], x[:, hq:hq + hk])
    torch.cuda.synchronize()
    assert torch.equal(bits(x[:, :hq].contiguous()), bits(out[:, hk:].contiguous()))
    assert torch.equal(bits(x[:, hq:hq + hk].contiguous()), bits(out[:, :hk].contiguous()))
    assert torch.equal(bits(x[:, hq + hk:].contiguous()), bits(keep[offset:][:x.numel()].view_as(x)[:, hq + hk:].contiguous()))
    assert torch.equal(bits(flat[:offset]), bits(keep[:offset])) and torch.equal(bits(flat[-5:]), bits(keep[-5:]))
    # an input broadcast over its heads
    one = randn(gen(9), n, 1, d, dtype=dtype).expand(n, hq, d)
    res = torch.empty((n, hq, d), dtype=DT[dtype], device="cuda")
    fcg.fcg_rope_apply(rope, dpos, one, res)
    torch.cuda.synchronize()
    assert all(torch.equal(res[:, 0], res[:, h]) for h in range(hq))


@pytest.mark.parametrize("pairs", [False, True])
def test_rope_apply_far_positions(pairs):
    """Any int32 position: the angle is taken in 64 bits.  Its rounding there, 2^-53 of p w and of p w / (2 pi),
    is another 2^31 2^-53 2 of a radian at most."""
    rope, w = make_rope(128, pairs, theta=1e6)
    pos = np.array([-2 ** 31, 2 ** 31 - 1, -1, 0, 1, 10 ** 9, 123456789, 2 ** 24 + 1])
    x = randn(gen(1), len(pos), 3, 128, dtype="f32")
    y = torch.empty_like(x)
    fcg.fcg_rope_apply(rope, torch.as_tensor(pos, dtype=torch.int32, device="cuda"), x, y)
    torch.cuda.synchronize()
    check_turned(y, turn64(x, pos, w, pairs), x, w, pairs, 1.0 + 2.0, "f32", "far")
    assert torch.equal(y[3], x[3])          # position 0 turns by nothing


@pytest.mark.parametrize("pairs", [False, True])
def test_rope_backward_is_the_gradient(pairs):
    """Against differences of the forward pass (linear in x: a difference is exact up to roundings) and as its
    transpose."""
    rope, w = make_rope(96, pairs, "linear", m=1.5)
    n, h, d = 9, 2, 128
    g = gen(3)
    x, e, gy = (randn(g, n, h, d, dtype="f32") for _ in range(3))
    pos = torch.arange(50, 50 + n, dtype=torch.int32, device="cuda")
    f = lambda t: (lambda y: (fcg.fcg_rope_apply(rope, pos, t, y), y)[1])(torch.empty_like(t))
    gx = torch.empty_like(x)
    fcg.fcg_rope_apply(rope, pos, gy, gx, flags=fcg.FCG_ROPE_BACKWARD)
    lhs = ((f(x + e) - f(x - e)).double() / 2 * gy).sum()
    rhs = (gx.double() * e).sum()
    # n h d products; each forward value is off by at most 2^-20 (|a| + |b|) m for inputs up to |x| + |e|
    size = float(((x.abs() + e.abs()).double().sum() + e.abs().double().sum()) * gy.abs().max())
    assert abs(float(lhs - rhs)) <= 2.0 ** -19 * 1.5 * 2 * size
    check_turned(gx, turn64(gy, np.arange(50, 50 + n), w, pairs, 1.5, -1.0), gy, w, pairs, 1.5, "f32", "gradient")


def test_rope_apply_replays_in_a_graph():
    rope, w = make_rope(64)
    x, y = randn(gen(5), 40, 4, 64), torch.zeros((40, 4, 64), dtype=torch.bfloat16, device="cuda")
    pos = torch.zeros(40, dtype=torch.int32, device="cuda")
    s = torch.cuda.Stream()
    gph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(gph, stream=s):
        fcg.fcg_rope_apply(rope, pos, x, y)
    for r in range(4):
        p = np.arange(40) * (r + 1) + 1000 * r
        pos.copy_(torch.as_tensor(p, dtype=torch.int32))
        x.copy_(randn(gen(50 + r), 40, 4, 64))
        gph.replay()
        torch.cuda.synchronize()
        check_turned(y, turn64(x, p, w, False), x, w, False, 1.0, "bf16", f"replay {r}")
        z = torch.empty_like(y)
        fcg.fcg_rope_apply(rope, pos, x, z)
        torch.cuda.synchronize()
        assert torch.equal(bits(y), bits(z))


# ------------------------------------------------------------------ append

def fill_memory(cache, dtype, value):
    K, V = cache_memory(cache, dtype)
    K.fill_(value), V.fill_(value)
    return K, V


SHAPES = [("bf16", 8, 2, 128), ("bf16", 4, 4, 64), ("f32", 4, 2, 64), ("f32", 8, 1, 128)]


@pytest.mark.parametrize("dtype,hq,hkv,d", SHAPES)
@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("form", ["own", "pairs-part", "half-scaled"])
def test_append_stores_encoded_rows_and_nothing_else(dtype, hq, hkv, d, page, form):
    L, S, T = 3, 4, 200
    rope, w, pairs, m = (None, freqs64(d, 1e4), False, 1.0) if form == "own" else \
        (*make_rope(d // 4, True, m=1.0), True, 1.0) if form == "pairs-part" else (*make_rope(d, False, "parts", m=1.2), False, 1.2)
    cache = fcg.Cache(fcg.model_desc(L, hq, hkv, d, 1e4, dtype), S, T, page, 60 if page else 0)
    K, V = fill_memory(cache, dtype, 7.0)
    want = {}
    rng = np.random.default_rng(7)
    # runs by value (ordered, reversed sequences), a scattered list, more runs than go by value, one token
    calls = [(np.repeat([2, 0], [50, 21]), np.r_[np.arange(5, 55), np.arange(0, 21)], 0, L)]
    sc = rng.permutation(150)
    calls.append((np.full(150, 1), sc, 1, 2))
    calls.append((np.full(100, 3), 2 * rng.permutation(100), 0, 1))
    calls.append((np.array([3]), np.array([199]), 2, 1))
    for ci, (seq, pos, l0, nl) in enumerate(calls):
        n = len(seq)
        x = randn(gen(ci), nl, n, hq + 2 * hkv, d, dtype=dtype)     # a fused projection's output
        q, k, v = x[:, :, :hq], x[:, :, hq:hq + hkv], x[:, :, hq + hkv:]
        qo = torch.full((nl, n, hq, d), float("nan"), dtype=DT[dtype], device="cuda")
        fcg.fcg_append(cache, l0, seq, pos, k, v, rope=rope, q=q, q_out=qo)
        torch.cuda.synchronize()
        check_turned(qo, turn64(q, pos, w, pairs, m), q, w, pairs, m, dtype, f"q of call {ci}")
        ref = turn64(k, pos, w, pairs, m)
        for l in range(nl):
            for s in np.unique(seq):
                at = torch.as_tensor(np.flatnonzero(seq == s), device="cuda")
                p = pos[seq == s]
                got = rows_of(cache, K, l0 + l, int(s), p)
                check_turned(got, ref[l][at], k[l][at], w, pairs, m, dtype, f"k of call {ci}")
                gv = rows_of(cache, V, l0 + l, int(s), p)
                assert torch.equal(bits(gv.contiguous()), bits(v[l][at].contiguous()))
                for i, pp in enumerate(p):
                    want[(l0 + l, int(s), int(pp))] = 1
    # every row that no call named still holds what it held
    n_rows = len(want) * hkv
    assert int((K != 7.0).any(-1).sum()) == n_rows and int((V != 7.0).any(-1).sum()) == n_rows
    cache.close()


@pytest.mark.parametrize("dtype,hq,hkv,d", SHAPES[:3])
@pytest.mark.parametrize("page", [0, 16])
def test_append_in_the_caches_form_equals_patch_prefill(dtype, hq, hkv, d, page):
    desc = fcg.model_desc(1, hq, hkv, d, 1e6, dtype)
    a, b = (fcg.Cache(desc, 2, 96, page, 12 if page else 0) for _ in range(2))
    n = 70
    seq, pos = np.repeat([0, 1], [40, 30]), np.r_[np.arange(40), np.arange(30)]
    q, k, v = randn(gen(1), n, hq, d, dtype=dtype), randn(gen(2), n, hkv, d, dtype=dtype), randn(gen(3), n, hkv, d, dtype=dtype)
    mem = [fill_memory(c, dtype, 0.0) for c in (a, b)]
    out, qo = torch.empty_like(q), torch.empty_like(q)
    fcg.fcg_patch_prefill(a, 0, seq, pos, q, k, v, out)
    fcg.fcg_append(b, 0, seq, pos, k, v, q=q, q_out=qo)
    # and the attention of both agrees: no prefix, every token over its own sequence
    o2 = torch.empty_like(q)
    fcg.fcg_prefix_attend(b, 0, -1, 0, seq, pos, qo, o2)
    torch.cuda.synchronize()
    assert torch.equal(bits(mem[0][0]), bits(mem[1][0])) and torch.equal(bits(mem[0][1]), bits(mem[1][1]))
    lim = 2e-2 if dtype == "bf16" else 1e-5
    assert float((out.float() - o2.float()).abs().max()) <= lim * max(1.0, float(out.float().abs().max()))
    # decoding goes on from an appended cache
    dq, dk, dv = (x[:2].clone() for x in (q, k, v))
    oa, ob = torch.empty_like(dq), torch.empty_like(dq)
    assert list(fcg.fcg_decode(a, 0, [0, 1], dq, dk, dv, oa)) == list(fcg.fcg_decode(b, 0, [0, 1], dq, dk, dv, ob))
    torch.cuda.synchronize()
    assert torch.equal(bits(oa), bits(ob))
    a.close(), b.close()


def test_append_replaces_reserves_and_reuses_pages():
    desc = fcg.model_desc(2, 4, 2, 64, 1e4, "bf16")
    c = fcg.Cache(desc, 2, 64, 16, 5)
    K, V = fill_memory(c, "bf16", 0.0)
    x = [randn(gen(i), 2, 20, 2, 64) for i in range(4)]
    pos = np.arange(10, 30)
    fcg.fcg_append(c, 0, np.zeros(20), pos, x[0], x[1])
    fcg.fcg_append(c, 0, np.zeros(20), pos, x[2], x[3], flags=fcg.FCG_REPLACE)
    torch.cuda.synchronize()
    for l in (0, 1):
        assert torch.equal(rows_of(c, V, l, 0, pos), x[3][l])
    fcg.fcg_append(c, 0, np.ones(40), np.arange(40), n_layers=2)        # reserved: pages 2, 3, 4
    fcg.fcg_cache_truncate(c, 0, 0)
    fcg.fcg_append(c, 0, np.ones(24), np.arange(40, 64), x[0][:, :1].expand(2, 24, 2, 64), x[1][:, :1].expand(2, 24, 2, 64))
    torch.cuda.synchronize()
    assert fcg.fcg_cache_export_layout(c, 1, 0)[0].tolist() == [2, 3, 4, 0]
    for l in (0, 1):
        assert torch.equal(rows_of(c, V, l, 1, np.arange(40, 64)), x[1][l, :1].expand(24, 2, 64))
    # pages mapped by the append are read by the decode that follows (the device table is current)
    q, k, v = randn(gen(8), 1, 4, 64), randn(gen(9), 1, 2, 64), randn(gen(10), 1, 2, 64)
    fcg.fcg_cache_truncate(c, 1, 63)
    out = torch.empty_like(q)
    fcg.fcg_decode(c, 0, [1], q, k, v, out)
    torch.cuda.synchronize()
    w = freqs64(64, 1e4)
    keys = rows_of(c, K, 0, 1, np.arange(64))
    ref = attend64(turn64(q, [63], w, False).to(torch.bfloat16), keys, rows_of(c, V, 0, 1, np.arange(64)), [63], 0)
    assert float((out.double() - ref[0]).abs().max()) <= 2e-2 + 2 ** -7 * float(ref[0].abs().max())
    c.close()


# ------------------------------------------------------------------ graft in a rotary form

@pytest.mark.parametrize("dtype,hq,hkv,d", SHAPES[:3])
@pytest.mark.parametrize("page,alias", [(0, False), (16, False), (16, True)])
@pytest.mark.parametrize("pairs,part", [(True, 1), (False, 4), (True, 4)])
def test_graft_rope(dtype, hq, hkv, d, page, alias, pairs, part):
    rope, w = make_rope(d // part, pairs, "parts", m=1.3)
    desc = fcg.model_desc(2, hq, hkv, d, 1e4, dtype)
    lens = [1, 70, 33, 64]
    lib = fcg.Library(desc, sum(lens), 4)
    segs = []
    for i, n in enumerate(lens):
        k, v = randn(gen(i), 2, n, hkv, d, dtype=dtype), randn(gen(10 + i), 2, n, hkv, d, dtype=dtype)
        fcg.fcg_lib_add_segment(lib, n, 5 * i, k, v)
        segs.append((k, v, 5 * i))
    for many in (False, True):          # the plan by value, and from memory (more than 32 items)
        S = 40 if many else 2
        c = fcg.Cache(desc, S, 240, page, 15 * S if page else 0, flags=fcg.FCG_ALIAS_V if alias else 0)
        K, V = fill_memory(c, dtype, 0.0)
        items = [(s, g, dst) for s in range(S) for g, dst in ((1, 0), (0, 71), (3, 100), (2, 15 + 164))]
        fcg.fcg_graft_rope(c, lib, rope, *map(list, zip(*items)))
        torch.cuda.synchronize()
        for s, g, dst in items[:4] + items[-4:]:
            k, v, src = segs[g]
            for l in (0, 1):
                pos = np.arange(dst, dst + lens[g])
                got = rows_of(c, K, l, s, pos)
                check_turned(got, turn64(k[l], np.full(lens[g], dst - src), w, pairs), k[l], w, pairs, 1.0, dtype, f"segment {g}")
                own = np.ones(lens[g], bool)
                if alias:
                    own = fcg.fcg_cache_export_v_alias(c, s)[pos // 16] < 0
                if own.any():
                    at = torch.as_tensor(np.flatnonzero(own), device="cuda")
                    assert torch.equal(rows_of(c, V, l, s, pos[own]), v[l][at])
        c.close()
    # at its source positions a segment is copied bit for bit
    c = fcg.Cache(desc, 1, 240, page, 15 if page else 0)
    K, V = fill_memory(c, dtype, 0.0)
    fcg.fcg_graft_rope(c, lib, rope, [0], [1], [5])
    torch.cuda.synchronize()
    assert torch.equal(rows_of(c, K, 1, 0, np.arange(5, 75)), segs[1][0][1])
    c.close(), lib.close()


def test_graft_rope_in_the_caches_form_agrees_with_graft():
    """The same frequencies through the handle: angles of another route, so the fp32 turns differ by a rounding."""
    desc = fcg.model_desc(2, 4, 2, 128, 1e6, "f32")
    rope, w = make_rope(128, theta=1e6)
    lib = fcg.Library(desc, 300, 1)
    k, v = randn(gen(0), 2, 300, 2, 128, dtype="f32"), randn(gen(1), 2, 300, 2, 128, dtype="f32")
    fcg.fcg_lib_add_segment(lib, 300, 17, k, v)
    mem = []
    for f in (lambda c: fcg.fcg_graft(c, lib, [0], [0], [900]), lambda c: fcg.fcg_graft_rope(c, lib, rope, [0], [0], [900])):
        c = fcg.Cache(desc, 1, 1200)
        m = fill_memory(c, "f32", 0.0)
        f(c)
        torch.cuda.synchronize()
        mem.append([t.clone() for t in m])
        c.close()
    assert torch.equal(mem[0][1], mem[1][1])
    assert float((mem[0][0] - mem[1][0]).abs().max()) <= 2.0 ** -20 * 2 * float(k.abs().max())
    lib.close()


# ------------------------------------------------------------------ attention over a shared prefix

class Shared:
    """A cache whose sequence `pseq` holds a prefix and whose others hold own tokens after it; K and V given as values."""

    def __init__(self, dtype, hq, hkv, d, page, prefix, own, seed, seqs=None, shuffle=True):
        S = len(own) + 1
        T = max(prefix + max(list(own) + [0]), 1) + 1
        self.dtype, self.P, self.own, self.pseq = dtype, prefix, own, len(own)
        n_pages = S * (-(-T // 16)) + 3
        self.cache = fcg.Cache(fcg.model_desc(2, hq, hkv, d, 1e4, dtype), S, T, page, n_pages if page else 0)
        self.mem = fill_memory(self.cache, dtype, float("nan"))      # what is not written must not matter
        g = gen(seed)
        seq = np.concatenate([np.full(prefix, self.pseq)] + [np.full(n, s) for s, n in enumerate(own)]).astype(np.int64)
        pos = np.concatenate([np.arange(prefix)] + [prefix + np.arange(n) for n in own]).astype(np.int64)
        order = np.random.default_rng(seed).permutation(len(seq)) if shuffle else np.arange(len(seq))
        for lo in range(0, len(seq), max(1, len(seq) // 3)):       # pages of the sequences end up interleaved
            at = np.sort(order[lo:lo + max(1, len(seq) // 3)])
            z = torch.zeros((len(at), hkv, d), dtype=DT[dtype], device="cuda")
            fcg.fcg_append(self.cache, 1, seq[at], pos[at], z, z)
        self.kv = {}
        for s in range(S):
            n, p0 = (prefix, 0) if s == self.pseq else (own[s], prefix)
            k, v = randn(g, n, hkv, d, dtype=dtype), randn(g, n, hkv, d, dtype=dtype)
            self.kv[s] = (k, v)
            self.put(s, np.arange(p0, p0 + n), k, v)

    def put(self, s, pos, k, v):
        if not len(pos):
            return
        pos = torch.as_tensor(pos, device="cuda")
        for m, x in zip(self.mem, (k, v)):
            if self.cache.page_size:
                pt = torch.as_tensor(fcg.fcg_cache_export_layout(self.cache, s, 1)[0].astype(np.int64), device="cuda")
                m[1][pt[pos // 16], :, pos % 16] = x
            else:
                m[1, s, :, pos] = x.transpose(0, 1)

    def joined(self, s):
        pk, pv = self.kv[self.pseq]
        k, v = self.kv[s]
        return (torch.cat([pk[:self.P], k]), torch.cat([pv[:self.P], v])) if s != self.pseq else (pk, pv)

    def check(self, seq, pos, q, out, lse, what, tokens=None):
        seq, pos = np.asarray(seq), np.asarray(pos)
        d = q.shape[-1]
        at = np.arange(len(seq)) if tokens is None else np.asarray(tokens)
        for s in np.unique(seq[at]):
            i = at[seq[at] == s]
            ii = torch.as_tensor(i, device="cuda")
            K, V = self.joined(int(s))
            ref = attend64(q[ii], K, V, pos[i], self.P)
            check_attend(out[ii], None if lse is None else lse[ii], ref, self.dtype, len(K), d, f"{what}, sequence {s}")


ATTN = [("bf16", 4, 1, 128), ("bf16", 8, 8, 64), ("bf16", 16, 1, 64), ("bf16", 16, 2, 128), ("bf16", 4, 2, 64),
        ("f32", 4, 2, 64), ("f32", 8, 1, 128), ("f32", 16, 1, 64), ("f32", 2, 2, 128)]


def run_shared(sh, seq, pos, seed, strided=False, scale=1.0):
    d, n = sh.cache.desc, len(seq)
    if strided:
        buf = randn(gen(seed), n, d.n_q_heads + 3, d.head_dim, dtype=sh.dtype)
        q = buf[:, 1:1 + d.n_q_heads]
        out = torch.full((n, 2 * d.n_q_heads, d.head_dim), float("nan"), dtype=DT[sh.dtype], device="cuda")[:, ::2]
    else:
        q = randn(gen(seed), n, d.n_q_heads, d.head_dim, dtype=sh.dtype) * scale
        out = torch.full_like(q, float("nan"))
    lse = torch.full((n, d.n_q_heads), float("nan"), device="cuda")
    fcg.fcg_prefix_attend(sh.cache, 1, sh.pseq if sh.P else -1, sh.P, seq, pos, q, out, lse)
    torch.cuda.synchronize()
    return q, out, lse


@pytest.mark.parametrize("dtype,hq,hkv,d", ATTN)
@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("prefix", [0, 1, 63, 129, 1000])
def test_prefix_attend_one_token_a_sequence(dtype, hq, hkv, d, page, prefix):
    own = [1, 17, 64, 200, 5, 16, 130] if prefix else [1, 17, 64, 200, 5, 16, 600]
    sh = Shared(dtype, hq, hkv, d, page, prefix, own, prefix + hq)
    seq = np.array([3, 0, 6, 1, 2, 5, 4])
    pos = np.array([prefix + own[s] - 1 for s in seq])
    q, out, lse = run_shared(sh, seq, pos, 1, strided=True)
    sh.check(seq, pos, q, out, lse, "decode")
    # fewer tokens than their sequences hold, one token alone, and the prefix alone (or no key at all)
    pos2 = np.maximum(prefix - 1, pos - 3)
    q, out, lse = run_shared(sh, seq, pos2, 2)
    sh.check(seq, pos2, q, out, lse, "earlier")
    q, out, lse = run_shared(sh, seq[:1], pos[:1], 3)
    sh.check(seq[:1], pos[:1], q, out, lse, "alone")
    q, out, lse = run_shared(sh, seq, np.full(7, prefix - 1), 4)
    sh.check(seq, np.full(7, prefix - 1), q, out, lse, "no own keys")
    if not prefix:
        assert not out.any() and torch.isinf(lse).all()
    sh.cache.close()


@pytest.mark.parametrize("dtype,hq,hkv,d", ATTN)
@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("prefix", [0, 77, 320])
def test_prefix_attend_several_tokens_a_sequence(dtype, hq, hkv, d, page, prefix):
    """Drafts of a few tokens, patch prompts that fill blocks of their own, one token, the same position twice."""
    own = [4, 200, 150, 1, 33]
    sh = Shared(dtype, hq, hkv, d, page, prefix, own, prefix + d)
    parts = [(0, range(prefix, prefix + 4)), (1, range(prefix + 40, prefix + 200)), (2, range(prefix, prefix + 140)),
             (3, [prefix]), (4, [prefix + 32, prefix + 32, prefix + 7, prefix + 30])]
    if prefix:
        parts.append((5, [prefix - 1]))      # the prefix's own sequence
    seq = np.concatenate([np.full(len(list(p)), s) for s, p in parts])
    pos = np.concatenate([np.array(list(p)) for _, p in parts])
    mix = np.random.default_rng(1).permutation(len(seq))
    seq, pos = seq[mix], pos[mix]
    q, out, lse = run_shared(sh, seq, pos, 5)
    some = np.unique(np.r_[np.flatnonzero(np.isin(seq, [0, 3, 4, 5])), np.arange(0, len(seq), 7)])
    sh.check(seq, pos, q, out, lse, "mixed", some)
    sh.cache.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [0, 16])
def test_prefix_attend_many_sequences_and_long_prefix(dtype, page):
    own = [1 + (37 * i) % 90 for i in range(70)]
    sh = Shared(dtype, 8, 2, 128, page, 5003, own, 11, shuffle=False)
    seq = np.arange(70)
    pos = np.array([5003 + n - 1 for n in own])
    q, out, lse = run_shared(sh, seq, pos, 6)
    sh.check(seq, pos, q, out, lse, "seventy", np.arange(0, 70, 9))
    # the same queries again: the same bits
    o2, l2 = torch.empty_like(out), torch.empty_like(lse)
    fcg.fcg_prefix_attend(sh.cache, 1, sh.pseq, sh.P, seq, pos, q, o2, l2)
    # in place, without lse
    fcg.fcg_prefix_attend(sh.cache, 1, sh.pseq, sh.P, seq, pos, q, q)
    torch.cuda.synchronize()
    assert torch.equal(bits(out), bits(o2)) and torch.equal(lse, l2) and torch.equal(bits(out), bits(q))
    sh.cache.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tokens", [2, 3, 40])
def test_prefix_attend_does_not_leak_masked_values(dtype, tokens):
    """Values (and keys) that are not finite at a position reach exactly the rows that see it."""
    P, own = 37, [tokens, 50]
    sh = Shared(dtype, 4, 2, 64, 16, P, own, 3)
    k, v = sh.kv[0]
    v[tokens - 1, 0, 5], v[tokens - 1, 1, 7] = float("inf"), float("nan")
    sh.put(0, np.arange(P, P + tokens), k, v)
    seq = np.r_[np.zeros(tokens, int), 1]
    pos = np.r_[P + np.arange(tokens), P + 20]
    q, out, lse = run_shared(sh, seq, pos, 8)
    last = tokens - 1
    keep = np.flatnonzero(~((seq == 0) & (pos == P + last)))
    sh.check(seq, pos, q, out, lse, "rows before it", keep)
    o = out[last].view(2, 2, 64)         # kv head, query of the group
    assert torch.isposinf(o[0, :, 5]).all() and torch.isnan(o[1, :, 7]).all()
    ok = torch.ones_like(o, dtype=torch.bool)
    ok[0, :, 5] = ok[1, :, 7] = False
    assert torch.isfinite(o[ok]).all()
    # a key that is not finite, seen by the last row only
    v[tokens - 1] = 1.0
    k[tokens - 1, 0, 3] = float("nan")
    sh.put(0, np.arange(P, P + tokens), k, v)
    q, out, lse = run_shared(sh, seq, pos, 9)
    sh.check(seq, pos, q, out, lse, "rows before the key", keep)
    assert torch.isnan(out[last, :2]).all() and torch.isfinite(out[last, 2:]).all()
    sh.cache.close()


def test_prefix_attend_large_scores_and_needles():
    """One key far above the others, in the prefix for some sequences and among the own keys for others."""
    P, own = 700, [90, 90, 90]
    sh = Shared("bf16", 4, 1, 128, 16, P, own, 4)
    q = randn(gen(1), 3, 4, 128)
    seq, pos = np.arange(3), np.full(3, P + 89)
    pk = sh.kv[sh.pseq][0]
    pk[500, 0] = q[0, 0] * 4
    sh.put(sh.pseq, np.arange(P), pk, sh.kv[sh.pseq][1])
    k1 = sh.kv[1][0]
    k1[40, 0] = q[1, 2] * 4
    sh.put(1, np.arange(P, P + 90), k1, sh.kv[1][1])
    out, lse = torch.empty_like(q), torch.empty((3, 4), device="cuda")
    fcg.fcg_prefix_attend(sh.cache, 1, sh.pseq, P, seq, pos, q, out, lse)
    torch.cuda.synchronize()
    sh.check(seq, pos, q, out, lse, "needles")
    assert float((out[0, 0] - sh.kv[sh.pseq][1][500, 0]).abs().max()) < 2e-2 * 4
    assert float((out[1, 2] - sh.kv[1][1][40, 0]).abs().max()) < 2e-2 * 4
    sh.cache.close()


def test_prefix_attend_reads_values_in_the_library():
    """A prefix grafted into an FCG_ALIAS_V cache: its values are read from the library."""
    desc = fcg.model_desc(1, 8, 2, 128, 1e4, "bf16")
    lib = fcg.Library(desc, 300, 1)
    k, v = randn(gen(0), 1, 300, 2, 128), randn(gen(1), 1, 300, 2, 128)
    fcg.fcg_lib_add_segment(lib, 300, 0, k, v)
    c = fcg.Cache(desc, 3, 400, 16, 60, flags=fcg.FCG_ALIAS_V)
    fcg.fcg_graft(c, lib, [2], [0], [0])
    assert (fcg.fcg_cache_export_v_alias(c, 2)[:18] >= 0).all()
    ok, ov = randn(gen(2), 2, 2, 128), randn(gen(3), 2, 2, 128)
    fcg.fcg_append(c, 0, [0, 1], [300, 300], ok, ov)
    q, out = randn(gen(4), 2, 8, 128), torch.empty((2, 8, 128), dtype=torch.bfloat16, device="cuda")
    fcg.fcg_prefix_attend(c, 0, 2, 300, [0, 1], [300, 300], q, out)
    torch.cuda.synchronize()
    w = freqs64(128, 1e4)
    for s in (0, 1):
        own = turn64(ok[s:s + 1], [300], w, False).to(torch.bfloat16)
        ref = attend64(q[s:s + 1], torch.cat([k[0], own]), torch.cat([v[0], ov[s:s + 1]]), [300], 300)
        check_attend(out[s:s + 1], None, ref, "bf16", 301, 128, f"sequence {s}")
    c.close(), lib.close()


# ------------------------------------------------------------------ all of them together

@pytest.mark.parametrize("dtype,page", [("bf16", 16), ("bf16", 0), ("f32", 16)])
def test_candidates_over_one_stitched_context(dtype, page):
    """Raw keys of two segments are encoded (apply) and put into a library, stitched in another order and at other
    places as the shared prefix (graft_rope), then three candidates prefill a prompt each and decode over it (append,
    prefix_attend), one of them retried in place; against one plain attention over the raw keys at their positions."""
    hq, hkv, d, L = 8, 2, 64, 2
    rope, w = make_rope(32, True, "parts", m=1.1)
    desc = fcg.model_desc(L, hq, hkv, d, 1e4, dtype)
    lens, dst, src = [150, 91], [91, 0], [40, 7]
    lib = fcg.Library(desc, sum(lens), 2)
    raw = []
    for i, n in enumerate(lens):
        k, v = randn(gen(i), L, n, hkv, d, dtype=dtype), randn(gen(9 + i), L, n, hkv, d, dtype=dtype)
        ke = torch.empty_like(k)
        fcg.fcg_rope_apply(rope, torch.arange(src[i], src[i] + n, dtype=torch.int32, device="cuda"), k=k, k_out=ke)
        fcg.fcg_lib_add_segment(lib, n, src[i], ke, v)
        raw.append((k, v))
    P = sum(lens)
    c = fcg.Cache(desc, 4, P + 80, page, 4 * (P + 80) // 16 if page else 0)
    fcg.fcg_graft_rope(c, lib, rope, [3, 3], [0, 1], dst)
    K = {s: torch.cat([raw[1][0], raw[0][0]], 1) for s in range(3)}
    V = {s: torch.cat([raw[1][1], raw[0][1]], 1) for s in range(3)}
    at = {s: P for s in range(3)}

    def step(counts, seed, replace=False):
        seq = np.repeat(np.arange(3), counts)
        pos = np.concatenate([at[s] + np.arange(m) for s, m in enumerate(counts)])
        n = len(seq)
        x = randn(gen(seed), L, n, hq + 2 * hkv, d, dtype=dtype)
        out = torch.empty((L, n, hq, d), dtype=DT[dtype], device="cuda")
        for l in range(L):
            q, k, v = x[l, :, :hq], x[l, :, hq:hq + hkv], x[l, :, hq + hkv:]
            qe = torch.empty((n, hq, d), dtype=DT[dtype], device="cuda")
            fcg.fcg_append(c, l, seq, pos, k, v, rope=rope, q=q, q_out=qe, flags=fcg.FCG_REPLACE if replace else 0)
            fcg.fcg_prefix_attend(c, l, 3, P, seq, pos, qe, out[l])
        torch.cuda.synchronize()
        for s in range(3):
            i = torch.as_tensor(np.flatnonzero(seq == s), device="cuda")
            K[s] = torch.cat([K[s][:, :at[s]], x[:, i, hq:hq + hkv]], 1)
            V[s] = torch.cat([V[s][:, :at[s]], x[:, i, hq + hkv:]], 1)
            for l in range(L):
                T = K[s].shape[1]
                enc = turn64(K[s][l], np.arange(T), w, True, 1.1)
                ref = attend64(turn64(x[l, i, :hq], pos[seq == s], w, True, 1.1), enc, V[s][l].double(), pos[seq == s], P)
                err = (out[l, i].double() - ref[0]).abs()
                # on top of the attention's own bound: keys and queries rounded once (twice for grafted keys: at the
                # source and after the turn), which moves each score by up to (2 + 1) half steps of sum |q k|
                moved = 3.1 * HALF_STEP[dtype] * ref[3][..., None] * 2.1 * ref[2]
                own = HALF_STEP[dtype] * ref[0].abs() + (2.02 * 2.0 ** -8 if dtype == "bf16" else 2.0 ** -15) * ref[2]
                assert bool((err <= moved * 1.5 + own + 1e-6).all()), (s, l, float((err - moved - own).max()))
        return counts

    step([20, 33, 1], 100)
    for s, m in enumerate([20, 33, 1]):
        at[s] += m
    step([1, 1, 1], 101)
    step([1, 1, 1], 102, replace=True)      # another try at the same positions
    for s in range(3):
        at[s] += 1
    step([4, 1, 2], 103)
    c.close(), lib.close()


# ------------------------------------------------------------------ graphs, streams, far offsets, block shapes

def test_append_and_attend_replay_in_graphs():
    """A decode step captured twice (two graphs that share the cache's workspace), replayed with new inputs between
    eager calls, one of which enlarges the workspace."""
    P, own = 900, [40 + 7 * i for i in range(8)]
    sh = Shared("bf16", 8, 2, 128, 16, P, own, 21)
    c, w = sh.cache, freqs64(64, 1e4)
    rope, _ = make_rope(64)
    seq, pos = np.arange(8), np.array([P + n - 1 for n in own])
    q, k, v = randn(gen(1), 8, 8, 128), randn(gen(2), 8, 2, 128), randn(gen(3), 8, 2, 128)
    qe, out, lse = torch.empty_like(q), torch.empty_like(q), torch.empty((8, 8), device="cuda")

    def step(stream=None):
        fcg.fcg_append(c, 1, seq, pos, k, v, rope=rope, q=q, q_out=qe, flags=fcg.FCG_REPLACE, stream=stream)
        fcg.fcg_prefix_attend(c, 1, sh.pseq, P, seq, pos, qe, out, lse, stream=stream)

    step()
    graphs = []
    for _ in range(2):
        s = torch.cuda.Stream()
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g, stream=s):
            step()
        graphs.append(g)
    many = np.repeat(np.arange(8), 30)
    mpos = np.concatenate([P + np.arange(n - 30, n) for n in own])
    mq = randn(gen(9), len(many), 8, 128)
    for r in range(5):
        for x, sd in ((q, 100), (k, 200), (v, 300)):
            x.copy_(randn(gen(sd + r), *x.shape))
        graphs[r % 2].replay()
        torch.cuda.synchronize()
        got = out.clone(), lse.clone(), qe.clone()
        for s in range(8):
            kk, vv = sh.kv[s]
            kk[own[s] - 1] = turn64(k[s:s + 1], pos[s:s + 1], w, False)[0].to(torch.bfloat16)
            vv[own[s] - 1] = v[s]
        sh.check(seq, pos, got[2], got[0], got[1], f"replay {r}")
        step()
        torch.cuda.synchronize()
        assert torch.equal(bits(out), bits(got[0])) and torch.equal(lse, got[1])
        if r == 1:      # a larger call takes a new workspace; the graphs keep theirs
            mo = torch.empty_like(mq)
            fcg.fcg_prefix_attend(c, 1, sh.pseq, P, many, mpos, mq, mo)
            torch.cuda.synchronize()
    sh.cache.close()


def test_prefix_attend_of_128_tokens_replays_in_a_graph():
    """The largest call that can be captured, over a prefix long enough for blocks of 256 rows."""
    P, own = 7001, [4 + 2 * i for i in range(32)]
    sh = Shared("bf16", 64, 8, 128, 16, P, own, 17, shuffle=False)
    seq = np.repeat(np.arange(32), 4)
    pos = np.concatenate([P + n - 4 + np.arange(4) for n in own])
    q = randn(gen(1), 128, 64, 128)
    out, lse = torch.empty_like(q), torch.empty((128, 64), device="cuda")

    def call():
        fcg.fcg_prefix_attend(sh.cache, 1, sh.pseq, P, seq, pos, q, out, lse)

    call()
    g, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=s):
        call()
    for r in range(3):
        q.copy_(randn(gen(50 + r), 128, 64, 128))
        out.fill_(float("nan")), lse.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        got = out.clone(), lse.clone()
        call()
        torch.cuda.synchronize()
        assert torch.equal(bits(out), bits(got[0])) and torch.equal(lse, got[1])
    sh.check(seq, pos, q, got[0], got[1], "replay", [0, 3, 65, 127])
    sh.cache.close()


def test_captures_that_need_an_upload_are_refused():
    sh = Shared("bf16", 8, 2, 64, 16, 100, [40] * 70, 5)
    c = sh.cache
    n = 70
    q, k, v = randn(gen(1), n, 8, 64), randn(gen(2), n, 2, 64), randn(gen(3), n, 2, 64)
    out = torch.empty_like(q)
    before = [fcg.fcg_cache_export_layout(c, s, 1) for s in (0, 70)]
    g, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=s):
        for call in (lambda: fcg.fcg_append(c, 1, [0], [0], k[:1], v[:1]),                               # maps a page
                     lambda: fcg.fcg_append(c, 1, np.arange(n), np.full(n, 139), k, v, flags=fcg.FCG_REPLACE),   # 70 runs
                     lambda: fcg.fcg_prefix_attend(c, 1, 70, 100, np.arange(n), np.full(n, 139), q, out),      # 70 sequences
                     lambda: fcg.fcg_prefix_attend(c, 1, 70, 100, [0, 1], [139, 139], q[:2], out[:2])):         # no workspace yet
            with pytest.raises(fcg.FcgError) as e:
                call()
            assert e.value.status == fcg.FCG_ESTATE
        out.zero_()
    for b, sq in zip(before, (0, 70)):
        now = fcg.fcg_cache_export_layout(c, sq, 1)
        assert b[1] == now[1] and np.array_equal(b[0], now[0]) and np.array_equal(b[2], now[2])
    g.replay()
    fcg.fcg_prefix_attend(c, 1, 70, 100, np.arange(n), np.full(n, 139), q, out)
    torch.cuda.synchronize()
    sh.check(np.arange(n), np.full(n, 139), q, out, None, "after", np.arange(0, n, 11))
    c.close()


def test_calls_on_another_stream_and_a_strided_result():
    sh = Shared("bf16", 4, 2, 64, 0, 130, [9, 70], 6)
    s = torch.cuda.Stream()
    big = torch.full((5, 9, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    q = randn(gen(1), 2, 4, 64)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        fcg.fcg_prefix_attend(sh.cache, 1, sh.pseq, 130, [0, 1], [138, 199], q, big[1:3, 2:6])
    s.synchronize()
    sh.check([0, 1], [138, 199], q, big[1:3, 2:6], None, "stream")
    rest = torch.ones((5, 9), dtype=torch.bool)
    rest[1:3, 2:6] = False
    assert bool((big[rest.cuda()] == 3.0).all())
    sh.cache.close()


def test_calls_larger_than_the_caches_equal_their_layers():
    """More than 256 MB of rows in one call (read and written past the caches): the bits of a call per layer."""
    L, n, hq, hkv, d = 9, 5001, 16, 8, 128
    rope, _ = make_rope(128, True, "ntk")
    c = fcg.Cache(fcg.model_desc(L, hq, hkv, d, 1e4, "bf16"), 2, n + 40, 16, 2 * (n + 40) // 16 + 2)
    mem = fill_memory(c, "bf16", 7.0)
    q, k, v = randn(gen(1), L, n, hq, d), randn(gen(2), L, n, hkv, d), randn(gen(3), L, n, hkv, d)
    assert q.numel() * 2 + k.numel() * 4 > 2 ** 28
    qo = torch.empty_like(q)
    pos = np.arange(17, 17 + n)
    dpos = torch.as_tensor(pos, dtype=torch.int32, device="cuda")
    fcg.fcg_append(c, 0, np.ones(n, int), pos, k, v, rope=rope, q=q, q_out=qo, n_layers=L)
    qq = torch.cat([q, q], 2)                       # 369 MB
    fcg.fcg_rope_apply(rope, dpos, qq, qq)
    torch.cuda.synchronize()
    assert torch.equal(bits(qq[:, :, :hq].contiguous()), bits(qo))
    for l in range(L):
        q1, k1 = torch.empty_like(q[l]), torch.empty_like(k[l])
        fcg.fcg_rope_apply(rope, dpos, q[l], q1, k[l], k1)
        torch.cuda.synchronize()
        assert torch.equal(bits(q1), bits(qo[l])) and torch.equal(bits(qq[l, :, hq:].contiguous()), bits(q1))
        assert torch.equal(bits(rows_of(c, mem[0], l, 1, pos)), bits(k1))
        assert torch.equal(bits(rows_of(c, mem[1], l, 1, pos)), bits(v[l]))
    c.close()


@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("hq,hkv,d", [(32, 2, 128), (16, 4, 64)])
def test_prefix_attend_blocks_of_many_rows(page, hq, hkv, d):
    """Calls whose rows fill blocks of 256 by themselves, with a rest that shares one, over whole prefix tiles and own
    keys that start inside a tile."""
    P = 2101
    own = [300, 128, 129, 200, 40]
    sh = Shared("bf16", hq, hkv, d, page, P, own, 31, shuffle=False)
    n = [128, 128, 77, 140, 3]
    seq = np.repeat(np.arange(5), n)
    pos = np.concatenate([P + own[s] - n[s] + np.arange(n[s]) for s in range(5)])
    q, out, lse = run_shared(sh, seq, pos, 7)
    some = np.unique(np.r_[np.arange(0, len(seq), 23), np.flatnonzero(seq == 4), np.cumsum(n) - 1])
    sh.check(seq, pos, q, out, lse, "blocks", some)
    sh.cache.close()


MANY = [128, 128, 77, 130, 128, 3]          # tokens of a sequence: blocks of 256 rows full and shared


@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("hq,hkv,d", [(32, 8, 128), (32, 8, 64), (16, 8, 64)])
def test_prefix_attend_blocks_of_256_rows(page, hq, hkv, d):
    """Calls large enough for blocks of 256 rows: fused and shared ones, tiles that hold the end of the prefix and the
    first own keys; also with scores so far apart that a few keys, in any tile, make the result."""
    P, own = 5003, [300, 128, 129, 200, 140, 90]
    sh = Shared("bf16", hq, hkv, d, page, P, own, 41, shuffle=False)
    seq = np.repeat(np.arange(6), MANY)
    pos = np.concatenate([P + own[s] - MANY[s] + np.arange(MANY[s]) for s in range(6)])
    some = np.unique(np.r_[np.arange(0, len(seq), 19), np.flatnonzero(seq == 5), np.cumsum(MANY) - 1])
    for scale in (1.0, 8.0):
        q, out, lse = run_shared(sh, seq, pos, 7, scale=scale)
        sh.check(seq, pos, q, out, lse, f"blocks, queries times {scale}", some)
    # values and keys of one sequence that are not finite reach exactly the rows that see them
    k, v = sh.kv[1]
    v[60, 0, 5], v[60, 1, 7], k[100, 2, 3] = float("inf"), float("nan"), float("nan")
    sh.put(1, np.arange(P, P + own[1]), k, v)
    q, out, lse = run_shared(sh, seq, pos, 8)
    v[60, 0, 5] = v[60, 1, 7] = k[100, 2, 3] = 0.0
    g, o = hq // hkv, out.view(len(seq), hkv, hq // hkv, d)
    at = np.flatnonzero(seq == 1)
    sees = torch.as_tensor(at[pos[at] >= P + 60], device="cuda")
    keys = torch.as_tensor(at[pos[at] >= P + 100], device="cuda")
    assert torch.isposinf(o[sees, 0, :, 5]).all() and torch.isnan(o[sees, 1, :, 7]).all() and torch.isnan(o[keys, 2]).all()
    assert torch.isnan(lse.view(len(seq), hkv, g)[keys, 2]).all()
    rest = torch.ones_like(o, dtype=torch.bool)
    rest[sees, 0, :, 5] = rest[sees, 1, :, 7] = rest[keys, 2] = False
    assert torch.isfinite(o[rest]).all()
    look = np.unique(np.r_[some[seq[some] != 1], at[::9][pos[at[::9]] < P + 100]])
    out2 = torch.zeros_like(o)
    out2[rest] = o[rest]
    for s in np.unique(seq[look]):
        t = look[seq[look] == s]
        K, V = sh.joined(int(s))
        ref = list(attend64(q[t], K, V, pos[t], P))
        ref[0] = ref[0] * rest[t].view(len(t), hq, d)
        check_attend(out2[t].view(len(t), hq, d), lse[t], ref, "bf16", len(K), d, f"around them, sequence {s}")
    sh.cache.close()


@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("hq,hkv,d,n_seq,P", [(64, 8, 128, 47, 2000), (64, 32, 64, 37, 0), (32, 16, 128, 64, 65),
                                              (128, 16, 64, 63, 300)])
def test_prefix_attend_more_own_items_than_run_at_once(page, hq, hkv, d, n_seq, P):
    """Small own parts that share blocks two by two: an odd number of them, of one to three tokens or none past the
    prefix, rows in one or two matrix tiles, lengths down to one key, values that are not finite behind a row's end."""
    rng = np.random.default_rng(n_seq)
    g = hq // hkv
    n = rng.integers(1, 4 if 3 * g <= 32 else 2, n_seq)
    n[rng.permutation(n_seq)[:max(0, int(n.sum()) - 128)]] = 1
    n = np.minimum(n, 128 // n_seq)
    own = [int(rng.integers(m, m + 1 if i % 5 == 0 else 150)) for i, m in enumerate(n)]
    sh = Shared("bf16", hq, hkv, d, page, P, own, 51, shuffle=False)
    seq = np.repeat(np.arange(n_seq), n)
    pos = np.concatenate([P + own[s] - n[s] + np.arange(n[s]) for s in range(n_seq)])
    if P:
        pos[np.flatnonzero(seq == 7)[0]] = P - 1        # the prefix only
    cut = 11                                            # its last key is not attended, and not finite
    own_cut = np.flatnonzero(seq == cut)
    if own[cut] > n[cut]:
        pos[own_cut] -= 1
        k, v = sh.kv[cut]
        k[-1], v[-1] = float("nan"), float("inf")
        sh.put(cut, np.arange(P, P + own[cut]), k, v)
    mix = rng.permutation(len(seq))
    seq, pos = seq[mix], pos[mix]
    for scale in (1.0, 8.0):
        q, out, lse = run_shared(sh, seq, pos, 5, scale=scale)
        sh.check(seq, pos, q, out, lse, f"queries times {scale}", np.arange(0, len(seq), 3))
    sh.cache.close()


def test_prefix_attend_one_item_a_row():
    """As many row blocks as fill the chip: no split, results written without a merge, in the queries' place too."""
    P, n = 4099, 32
    sh = Shared("bf16", 32, 8, 128, 16, P, [64 + i for i in range(n)], 43, shuffle=False)
    seq = np.repeat(np.arange(n), 64)
    pos = np.concatenate([P + i + np.arange(64) for i in range(n)])
    some = np.unique(np.r_[np.arange(0, len(seq), 97), len(seq) - 1])
    for scale in (1.0, 8.0):
        q, out, lse = run_shared(sh, seq, pos, 3, scale=scale)
        sh.check(seq, pos, q, out, lse, f"direct, queries times {scale}", some)
        fcg.fcg_prefix_attend(sh.cache, 1, sh.pseq, P, seq, pos, q, q)
        torch.cuda.synchronize()
        assert torch.equal(bits(q), bits(out))
    sh.cache.close()


def test_prefix_attend_blocks_of_256_rows_read_values_in_the_library():
    """The same over a prefix of two grafted segments whose values stay in the library, but for the page they share."""
    lens, hq, hkv, d = [2503, 2500], 32, 8, 128
    P = sum(lens)
    desc = fcg.model_desc(1, hq, hkv, d, 1e4, "bf16")
    lib = fcg.Library(desc, P, 2)
    k, v = randn(gen(0), P, hkv, d), randn(gen(1), P, hkv, d)
    for p0, n in ((0, lens[0]), (lens[0], lens[1])):        # at their own positions: keys as they are
        fcg.fcg_lib_add_segment(lib, n, p0, k[None, p0:p0 + n].contiguous(), v[None, p0:p0 + n].contiguous())
    c = fcg.Cache(desc, 7, P + 140, 16, 7 * (P + 140) // 16, flags=fcg.FCG_ALIAS_V)
    fcg.fcg_graft(c, lib, [6, 6], [1, 0], [lens[0], 0])
    alias = fcg.fcg_cache_export_v_alias(c, 6)[:P // 16]
    assert (alias >= 0).sum() == P // 16 - 1
    seq = np.repeat(np.arange(6), MANY)
    pos = np.concatenate([P + np.arange(n) for n in MANY])
    ok, ov = torch.zeros((len(seq), hkv, d), dtype=torch.bfloat16, device="cuda"), randn(gen(3), len(seq), hkv, d)
    fcg.fcg_append(c, 0, seq, pos, ok, ov)
    q = randn(gen(4), len(seq), hq, d) * 8.0
    out = torch.full_like(q, float("nan"))
    fcg.fcg_prefix_attend(c, 0, 6, P, seq, pos, q, out)
    torch.cuda.synchronize()
    for t in range(0, len(seq), 17):
        own = torch.as_tensor(np.flatnonzero(seq == seq[t]), device="cuda")
        K, V = torch.cat([k, ok[own]]), torch.cat([v, ov[own]])
        check_attend(out[t:t + 1], None, attend64(q[t:t + 1], K, V, pos[t:t + 1], P), "bf16", len(K), d, f"token {t}")
    c.close(), lib.close()


def test_offsets_past_32_bits():
    """Pages, sequences and rows whose element offsets pass 2^31."""
    desc = fcg.model_desc(1, 8, 8, 128, 1e4, "bf16")
    n0 = 2 ** 31 // (8 * 128) + 64                     # positions before the ones looked at
    for page in (0, 16):
        if page:
            c = fcg.Cache(desc, 3, n0, 16, n0 // 16 + 40)
            fcg.fcg_append(c, 0, np.zeros(n0, np.int32), np.arange(n0, dtype=np.int32))      # reserved
        else:
            c = fcg.Cache(desc, 36, 65536)
        a, b = (1, 2) if page else (34, 35)
        P = 150
        pk, pv = randn(gen(1), P, 8, 128), randn(gen(2), P, 8, 128)
        ok, ov = randn(gen(3), 3, 8, 128), randn(gen(4), 3, 8, 128)
        fcg.fcg_append(c, 0, np.full(P, a), np.arange(P), pk, pv)
        fcg.fcg_append(c, 0, np.full(3, b), P + np.arange(3), ok, ov)
        q, out = randn(gen(5), 3, 8, 128), torch.empty((3, 8, 128), dtype=torch.bfloat16, device="cuda")
        fcg.fcg_prefix_attend(c, 0, a, P, np.full(3, b), P + np.arange(3), q, out)
        torch.cuda.synchronize()
        w = freqs64(128, 1e4)
        K = torch.cat([turn64(pk, np.arange(P), w, False), turn64(ok, P + np.arange(3), w, False)]).to(torch.bfloat16)
        V = torch.cat([pv, ov])
        ref = attend64(q, K, V, P + np.arange(3), P)
        # the stored keys may be one rounding from K: each score by another half step of sum |q k|
        err = (out.double() - ref[0]).abs()
        tol = 2.0 ** -8 * ref[0].abs() + (2.02 * 2.0 ** -8 + 2.0 ** -13) * ref[2]
        assert bool((err <= tol).all()), float((err - tol).max())
        c.close()
    n, h = 265000, 64
    x = torch.empty((n, h, 128), dtype=torch.bfloat16, device="cuda")
    x[-5:] = randn(gen(6), 5, h, 128)
    x[:5] = randn(gen(7), 5, h, 128)
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    rope, w = make_rope(128, True)
    y = torch.empty_like(x)
    fcg.fcg_rope_apply(rope, pos, x, y)
    torch.cuda.synchronize()
    for sl, p in ((slice(0, 5), np.arange(5)), (slice(n - 5, n), np.arange(n - 5, n))):
        check_turned(y[sl], turn64(x[sl], p, w, True), x[sl], w, True, 1.0, "bf16", "far rows")

"""Rotary handles, append and prefix attention without a GPU: frequencies, layout, refusals."""
import ctypes

import numpy as np
import pytest

from opsutil import freqs64
from paper_2606_13097_amd import fcg

E = fcg


def refuses(status, f, *a, **k):
    with pytest.raises(fcg.FcgError) as e:
        f(*a, **k)
    assert e.value.status == status, str(e.value)


@pytest.mark.parametrize("rot", [16, 48, 64, 112, 128])
@pytest.mark.parametrize("kind,code", [("plain", 0), ("linear", 1), ("ntk", 2), ("parts", 3)])
def test_frequencies_follow_their_formula(rot, kind, code):
    r = fcg.fcg_rope_create(rot, 1e6, scaling=code, factor=4.0, orig_tokens=32768, low_turns=1.0, high_turns=32.0)
    w = fcg.fcg_rope_frequencies(r)
    ref = freqs64(rot, 1e6, kind, 4.0, 32768.0)
    np.testing.assert_allclose(w, ref, rtol=1e-13)
    if kind == "parts":      # the fastest pair keeps its frequency, the slowest is interpolated
        assert w[0] == 1.0
        assert rot < 48 or abs(w[-1] * 4 / freqs64(rot, 1e6)[-1] - 1) < 1e-13
    g = fcg.fcg_rope_create(rot, scaling=E.FCG_ROPE_GIVEN, freqs=w)
    assert np.array_equal(fcg.fcg_rope_frequencies(g), w)


def test_rope_refusals():
    ok = dict(rotary_dim=64, theta=1e4)
    for bad in (dict(rotary_dim=0), dict(rotary_dim=8), dict(rotary_dim=24), dict(rotary_dim=144), dict(rotary_dim=-16),
                dict(layout=2), dict(layout=-1), dict(scaling=5), dict(scaling=-1), dict(theta=1.0), dict(theta=float("nan")),
                dict(theta=float("inf")), dict(attn_factor=0.0), dict(attn_factor=float("nan")),
                dict(scaling=1, factor=0.5), dict(scaling=2, factor=float("inf")), dict(scaling=3, factor=2.0),
                dict(scaling=3, factor=2.0, orig_tokens=100, low_turns=4.0, high_turns=4.0),
                dict(scaling=3, factor=2.0, orig_tokens=100, low_turns=-1.0), dict(scaling=4),
                dict(scaling=4, freqs=[float("inf")] + [0.0] * 31)):
        refuses(E.FCG_EINVAL, fcg.fcg_rope_create, **{**ok, **bad})
    with pytest.raises(ValueError):
        fcg.fcg_rope_create(64, scaling=4, freqs=[1.0] * 31)
    assert fcg._L.fcg_rope_create(None, None) == E.FCG_EINVAL
    assert fcg._L.fcg_rope_frequencies(None, None) == E.FCG_EINVAL
    assert fcg._L.fcg_rope_destroy(None) == E.FCG_OK


def V(data=64, layer=0, token=256, head=64):
    return fcg.TensorView(data, layer, token, head)


def apply(rope, dt=1, d=64, layers=1, n=2, pos=64, hq=4, q=None, qo=None, hk=0, k=None, ko=None, flags=0):
    r = [None if t is None else ctypes.byref(t) for t in (q, qo, k, ko)]
    fcg._check(fcg._L.fcg_rope_apply(None if rope is None else rope.h, dt, d, layers, n, pos, hq, r[0], r[1], hk, r[2], r[3],
                                     flags, None))


def test_apply_refusals_reach_no_kernel():
    r64, r128 = fcg.fcg_rope_create(64), fcg.fcg_rope_create(128)
    v = V()
    for bad in (dict(rope=None), dict(dt=2), dict(d=96), dict(d=32), dict(rope=r128), dict(layers=-1), dict(n=-1),
                dict(hq=-1), dict(hq=4097), dict(flags=2), dict(pos=None), dict(qo=None), dict(q=V(None)), dict(qo=V(None)),
                dict(q=V(token=-1)), dict(qo=V(head=-64)),
                dict(qo=V(token=255)), dict(qo=V(head=63)), dict(qo=V(token=0)), dict(layers=2),       # rows that meet
                dict(layers=2, qo=V(layer=511)), dict(q=V(token=512)), dict(qo=V(token=512))):            # in place, other strides
        refuses(E.FCG_EINVAL, apply, **{**dict(rope=r64, q=v, qo=v), **bad})
    # nothing to do: no launch, whatever the pointers
    apply(r64, n=0, q=V(None), qo=V(None), pos=None)
    apply(r64, hq=0, pos=None)
    apply(r64, layers=0, q=v, qo=v)


def layout_cache(n_seqs=3, max_tokens=100, page=16, n_pages=24, L=2, flags=0):
    d = fcg.model_desc(L, 4, 2, 64, 1e4, "bf16")
    return fcg.Cache(d, n_seqs, max_tokens, page, n_pages, flags=fcg.FCG_LAYOUT_ONLY | flags)


@pytest.mark.parametrize("page", [0, 16])
def test_append_places_tokens_and_leaves_holes(page):
    c = layout_cache(page=page)
    fcg.fcg_append(c, 0, [1, 0, 1], [40, 7, 41], n_layers=2)
    for layer in (0, 1):
        pt, n, wr = fcg.fcg_cache_export_layout(c, 1, layer)
        assert n == 42 and np.flatnonzero(wr).tolist() == [40, 41]
        if page:
            assert pt.tolist() == [-1, -1, 1, -1, -1, -1, -1]     # (sequence, page) order: sequence 0 took page 0
    # attention calls refuse the hole, and a later append fills it
    refuses(E.FCG_EHOLE, fcg.fcg_decode, c, 0, [1], None, None, None, None)
    refuses(E.FCG_EHOLE, fcg.fcg_patch_prefill, c, 0, [1], [42], None, None, None, None)
    fcg.fcg_append(c, 0, np.ones(40), np.arange(40))
    assert fcg.fcg_decode(c, 0, [1], None, None, None, None).tolist() == [42]
    assert fcg.fcg_cache_export_layout(c, 1, 1)[2].sum() == 2


def test_append_refusals_change_nothing():
    c = layout_cache()
    fcg.fcg_append(c, 1, [0, 0], [5, 6])
    before = [fcg.fcg_cache_export_layout(c, 0, l) for l in (0, 1)]
    def bad(status, *a, **k):
        refuses(status, fcg.fcg_append, c, *a, **k)
        for b, l in zip(before, (0, 1)):
            now = fcg.fcg_cache_export_layout(c, 0, l)
            assert b[1] == now[1] and np.array_equal(b[0], now[0]) and np.array_equal(b[2], now[2])
    bad(E.FCG_ERANGE, 2, [0], [1])
    bad(E.FCG_ERANGE, -1, [0], [1])
    bad(E.FCG_ERANGE, 1, [0], [1], n_layers=2)
    bad(E.FCG_EINVAL, 0, [0], [1], n_layers=-1)
    bad(E.FCG_ERANGE, 0, [3], [1])
    bad(E.FCG_ERANGE, 0, [-1], [1])
    bad(E.FCG_ERANGE, 0, [0], [100])
    bad(E.FCG_ERANGE, 0, [0], [-1])
    bad(E.FCG_EOVERLAP, 0, [0, 0], [1, 1])
    bad(E.FCG_EOVERLAP, 0, [0, 0], [1, 1], flags=E.FCG_REPLACE)
    bad(E.FCG_EOVERLAP, 1, [0], [6])
    bad(E.FCG_EOVERLAP, 0, [0], [6], n_layers=2)            # written in layer 1 only
    bad(E.FCG_EINVAL, 0, [0], [1], flags=2)
    bad(E.FCG_EINVAL, 0, [0], [1], rope=fcg.fcg_rope_create(128))    # heads of 64
    assert fcg._L.fcg_append(None, 0, 1, 0, None, None, None, None, None, None, None, 0, None) == E.FCG_EINVAL
    # written over with FCG_REPLACE, in a layer where it is new as well
    fcg.fcg_append(c, 0, [0], [6], n_layers=2, flags=E.FCG_REPLACE)
    assert fcg.fcg_cache_export_layout(c, 0, 0)[1] == 7
    # out of pages
    c = layout_cache(n_pages=2)
    refuses(E.FCG_ENOMEM, fcg.fcg_append, c, 0, [0, 0, 0], [0, 16, 32])
    fcg.fcg_append(c, 0, [0, 0], [0, 32])
    # no tokens, no layers
    fcg.fcg_append(c, 0, [], [])
    fcg.fcg_append(c, 0, [0], [64], n_layers=0)


def test_append_does_not_replace_values_read_from_the_library():
    d = fcg.model_desc(2, 4, 2, 64, 1e4, "bf16")
    c = layout_cache(flags=fcg.FCG_ALIAS_V)
    lib = fcg.Library(d, 64, 1, flags=fcg.FCG_LAYOUT_ONLY)
    fcg.fcg_lib_add_segment(lib, 40, 0)
    fcg.fcg_graft(c, lib, [0], [0], [4])        # pages 1 and 2 lie inside positions 4 .. 43
    for p in (16, 31, 32, 40):
        refuses(E.FCG_ESTATE if p < 32 else E.FCG_EOVERLAP, fcg.fcg_append, c, 0, [0], [p],
                flags=E.FCG_REPLACE if p < 32 else 0)
    fcg.fcg_append(c, 0, [0], [5], flags=E.FCG_REPLACE)
    fcg.fcg_append(c, 0, [0], [43], flags=E.FCG_REPLACE)
    fcg.fcg_cache_truncate(c, 0, 20)            # splits page 1: its values are its own now
    fcg.fcg_append(c, 0, [0], [18], flags=E.FCG_REPLACE)


def attend(c, pseq, plen, seq, pos, layer=0):
    fcg.fcg_prefix_attend(c, layer, pseq, plen, seq, pos, None, None)


def test_prefix_attend_checks_what_it_would_read():
    c = layout_cache()
    fcg.fcg_append(c, 0, np.full(30, 2), np.arange(30))
    fcg.fcg_append(c, 0, [0, 0, 1], [25, 26, 25])
    attend(c, 2, 25, [0, 1, 0, 1], [26, 25, 25, 24])
    attend(c, 2, 30, [2, 0], [29, 29])                      # the prefix alone
    attend(c, 2, 10, [2], [29])                             # the prefix's own sequence goes on
    attend(c, -1, 0, [0], [-1])                             # nothing at all
    attend(c, 9, 0, [2], [29])                              # no prefix: its sequence is not looked at
    attend(c, 2, 25, [], [])
    for status, a in ((E.FCG_EHOLE, (2, 31, [0], [30])), (E.FCG_EHOLE, (2, 24, [0], [26])),
                      (E.FCG_EHOLE, (2, 25, [1], [26])), (E.FCG_EHOLE, (2, 25, [0, 1, 0], [25, 25, 27])),
                      (E.FCG_EHOLE, (0, 1, [0], [0])), (E.FCG_EHOLE, (-1, 0, [0], [0])),
                      (E.FCG_ERANGE, (3, 25, [0], [25])), (E.FCG_ERANGE, (-1, 25, [0], [25])),
                      (E.FCG_ERANGE, (2, -1, [0], [25])), (E.FCG_ERANGE, (2, 101, [0], [100])),
                      (E.FCG_ERANGE, (2, 25, [0], [23])), (E.FCG_ERANGE, (2, 25, [3], [25])),
                      (E.FCG_ERANGE, (2, 25, [0], [100])), (E.FCG_ERANGE, (-1, 0, [0], [-2]))):
        refuses(status, attend, c, *a)
    refuses(E.FCG_ERANGE, attend, c, 2, 25, [0], [25], layer=2)
    refuses(E.FCG_EHOLE, attend, c, 2, 25, [0], [25], layer=1)
    assert fcg._L.fcg_prefix_attend(c.h, 0, 2, 25, -1, None, None, None, None, None, None) == E.FCG_EINVAL
    assert fcg._L.fcg_prefix_attend(c.h, 0, 2, 25, 1, None, None, None, None, None, None) == E.FCG_EINVAL


def test_graft_rope_refusals():
    d = fcg.model_desc(2, 4, 2, 64, 1e4, "bf16")
    c, lib = layout_cache(), fcg.Library(d, 64, 1, flags=fcg.FCG_LAYOUT_ONLY)
    fcg.fcg_lib_add_segment(lib, 40, 0)
    r = fcg.fcg_rope_create(32)
    refuses(E.FCG_EINVAL, fcg.fcg_graft_rope, c, lib, fcg.fcg_rope_create(128), [0], [0], [0])
    assert fcg._L.fcg_graft_rope(c.h, lib.h, None, 0, None, None, None, None) == E.FCG_EINVAL
    refuses(E.FCG_ERANGE, fcg.fcg_graft_rope, c, lib, r, [0], [1], [0])
    refuses(E.FCG_ERANGE, fcg.fcg_graft_rope, c, lib, r, [0], [0], [61])
    fcg.fcg_graft_rope(c, lib, r, [0], [0], [60])
    refuses(E.FCG_EOVERLAP, fcg.fcg_graft_rope, c, lib, r, [0], [0], [25])
    assert fcg.fcg_cache_export_layout(c, 0, 1)[1] == 100

"""Attention weight per position and eviction without a GPU: refusals, layouts."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2606_13097_amd import fcg

E = fcg


def refuses(status, f, *a, **k):
    with pytest.raises(fcg.FcgError) as e:
        f(*a, **k)
    assert e.value.status == status, str(e.value)


def weights(c, layer=0, pre=0, P=0, seq=(0,), pos=(0,), n=None, q=None, lse=None, w=None, flags=0, arrays=True):
    s, p = np.array(seq, dtype=np.int32), np.array(pos, dtype=np.int32)
    fcg._check(fcg._L.fcg_attend_weights(None if c is None else c.h, layer, pre, P, len(s) if n is None else n,
                                         fcg._p(s) if arrays else None, fcg._p(p), None if q is None else ctypes.byref(q),
                                         lse, w, flags, None))


def test_weights_refusals():
    c = fcg.Cache(fcg.model_desc(2, 4, 2, 64, 1e4, "bf16"), 3, 64, flags=fcg.FCG_LAYOUT_ONLY)
    fcg.fcg_append(c, 0, [0] * 40 + [1] * 10, list(range(40)) + list(range(30, 40)), n_layers=2)
    fcg.fcg_append(c, 0, [2], [0])
    weights(c, P=30, seq=[1, 1, 0], pos=[39, 29, 35])
    weights(c, n=0)
    refuses(E.FCG_EINVAL, weights, None)
    refuses(E.FCG_EINVAL, weights, c, n=-1)
    refuses(E.FCG_EINVAL, weights, c, arrays=False)
    refuses(E.FCG_EINVAL, weights, c, flags=2)
    refuses(E.FCG_EINVAL, weights, c, n=1 << 24)
    refuses(E.FCG_ERANGE, weights, c, layer=2)
    refuses(E.FCG_ERANGE, weights, c, layer=-1)
    refuses(E.FCG_ERANGE, weights, c, P=65)
    refuses(E.FCG_ERANGE, weights, c, P=1, pre=3)
    refuses(E.FCG_ERANGE, weights, c, seq=[3])
    refuses(E.FCG_ERANGE, weights, c, pos=[64])
    refuses(E.FCG_ERANGE, weights, c, P=30, pos=[28])
    refuses(E.FCG_EHOLE, weights, c, pos=[40])
    refuses(E.FCG_EHOLE, weights, c, seq=[1], pos=[35])
    refuses(E.FCG_EHOLE, weights, c, P=41, pos=[41])
    refuses(E.FCG_EHOLE, weights, c, layer=1, seq=[2], pos=[0])


def test_weights_checks_of_the_binding():
    c = fcg.Cache(fcg.model_desc(1, 4, 2, 64, 1e4, "bf16"), 1, 32, flags=fcg.FCG_LAYOUT_ONLY)
    with pytest.raises(ValueError):
        fcg.fcg_attend_weights(c, 0, 0, 0, [0, 1], [0], None, None, None)
    with pytest.raises(ValueError):     # not on a GPU
        fcg.fcg_attend_weights(c, 0, 0, 0, [0], [0], torch.zeros(1, 4, 64, dtype=torch.bfloat16), torch.zeros(1, 4),
                               torch.zeros(1, 2, 32))


def evict(c, src=(0,), dst=(0,), keep=(1,), first=0, recent=0, rope=None, w=None, n=None, arrays=True):
    a, b, k = (np.array(x, dtype=np.int32) for x in (src, dst, keep))
    fcg._check(fcg._L.fcg_evict(None if c is None else c.h, len(a) if n is None else n, fcg._p(a) if arrays else None,
                                fcg._p(b), fcg._p(k), first, recent, None if rope is None else rope.h, w, None, None))


def layout(c):
    out = []
    for s in range(c.n_seqs):
        for l in range(c.desc.n_layers):
            pt, n, wr = fcg.fcg_cache_export_layout(c, s, l)
            out.append((None if pt is None else pt.tolist(), n, wr.tolist()))
    return out


def test_evict_refusals_change_nothing():
    c = fcg.Cache(fcg.model_desc(2, 4, 2, 64, 1e4, "bf16"), 6, 64, 16, 12, fcg.FCG_LAYOUT_ONLY)
    fcg.fcg_append(c, 0, [0] * 60 + [1] * 33, list(range(60)) + list(range(33)), n_layers=2)   # 4 + 3 pages
    fcg.fcg_append(c, 0, [2] * 5, range(5))                              # layer 0 alone
    fcg.fcg_append(c, 0, [3] * 5, range(1, 6), n_layers=2)               # position 0 is a hole
    fcg.fcg_append(c, 0, [4] * 20, range(20), n_layers=2)                # 2 pages: 1 free
    before = layout(c)
    refuses(E.FCG_EINVAL, evict, None)
    refuses(E.FCG_EINVAL, evict, c, n=-1)
    refuses(E.FCG_EINVAL, evict, c, arrays=False)
    refuses(E.FCG_EINVAL, evict, c, first=-1)
    refuses(E.FCG_EINVAL, evict, c, recent=-1)
    refuses(E.FCG_EINVAL, evict, c, rope=fcg.fcg_rope_create(128))
    refuses(E.FCG_EINVAL, evict, c, src=[0, 1], dst=[5, 5], keep=[1, 1])
    refuses(E.FCG_EINVAL, evict, c, src=[0, 1], dst=[0, 0], keep=[1, 1])
    refuses(E.FCG_EINVAL, evict, c, src=[0, 0], dst=[0, 5], keep=[1, 1])
    refuses(E.FCG_EINVAL, evict, c, src=[0, 1], dst=[1, 5], keep=[1, 1])
    refuses(E.FCG_ERANGE, evict, c, src=[6])
    refuses(E.FCG_ERANGE, evict, c, dst=[-1])
    refuses(E.FCG_ERANGE, evict, c, keep=[65])
    refuses(E.FCG_ERANGE, evict, c, keep=[-1])
    refuses(E.FCG_ESTATE, evict, c, src=[2], dst=[2])
    refuses(E.FCG_EHOLE, evict, c, src=[3], dst=[5])
    refuses(E.FCG_ENOMEM, evict, c, src=[0], dst=[5], keep=[17])         # 2 pages
    refuses(E.FCG_ENOMEM, evict, c, src=[0, 1], dst=[4, 5], keep=[33, 16])
    assert layout(c) == before
    evict(c, n=0)
    assert layout(c) == before


@pytest.mark.parametrize("page", [0, 16])
def test_evict_layouts(page):
    """In place the tail goes and its pages return; another sequence is emptied first and its pages serve again."""
    c = fcg.Cache(fcg.model_desc(2, 4, 2, 64, 1e4, "bf16"), 4, 64, page, 9 if page else 0, fcg.FCG_LAYOUT_ONLY)
    fcg.fcg_append(c, 0, [0] * 60 + [1] * 33, list(range(60)) + list(range(33)), n_layers=2)
    fcg.fcg_append(c, 0, [2] * 2, [5, 30], n_layers=2)                   # a target may have holes: pages 7, 8
    evict(c, src=[0, 1], dst=[2, 1], keep=[31, 17])
    if page:
        assert fcg.fcg_cache_export_layout(c, 2, 0)[0].tolist() == [7, 8, -1, -1]
        assert fcg.fcg_cache_export_layout(c, 1, 0)[0].tolist() == [4, 5, -1, -1]
    for s, n in ((0, 60), (1, 17), (2, 31)):
        for l in (0, 1):
            _, got, wr = fcg.fcg_cache_export_layout(c, s, l)
            assert got == n and wr.tolist() == [1] * n + [0] * (64 - n)
    evict(c, src=[0], dst=[3], keep=[0])
    assert fcg.fcg_cache_export_layout(c, 3, 0)[1] == 0
    evict(c, src=[3], dst=[2], keep=[9])                                 # an empty source empties the target
    assert fcg.fcg_cache_export_layout(c, 2, 1)[1] == 0
    evict(c, src=[0], dst=[0], keep=[64])                                # fewer than asked for: all stay
    assert fcg.fcg_cache_export_layout(c, 0, 1)[1] == 60
    fcg.fcg_append(c, 0, [1], [17], n_layers=2)                          # and it goes on from there
    assert fcg.fcg_cache_export_layout(c, 1, 1)[1] == 18


def test_evict_in_place_refuses_values_in_the_library():
    desc = fcg.model_desc(1, 4, 2, 64, 1e4, "bf16")
    lib = fcg.Library(desc, 64, 2, flags=fcg.FCG_LAYOUT_ONLY)
    fcg.fcg_lib_add_segment(lib, 40, 0)
    c = fcg.Cache(desc, 2, 64, 16, 8, fcg.FCG_LAYOUT_ONLY | fcg.FCG_ALIAS_V)
    fcg.fcg_graft(c, lib, [0], [0], [0])
    refuses(E.FCG_ESTATE, evict, c, keep=[10])
    evict(c, dst=[1], keep=[10])
    assert fcg.fcg_cache_export_v_alias(c, 1).tolist() == [-1] * 4
    fcg.fcg_graft(c, lib, [1], [0], [16])
    evict(c, dst=[1], keep=[10])                                         # emptied: its values leave the library
    assert fcg.fcg_cache_export_v_alias(c, 1).tolist() == [-1] * 4


@pytest.mark.parametrize("layers,heads,status", [(255, 4096, 0), (255, 8192, E.FCG_EINVAL), (1, 32768, E.FCG_EINVAL)])
def test_evict_refuses_more_heads_than_a_launch_takes(layers, heads, status):
    c = fcg.Cache(fcg.model_desc(layers, heads, heads, 64, 1e4, "bf16"), 1, 8, flags=fcg.FCG_LAYOUT_ONLY)
    fcg.fcg_append(c, 0, [0] * 3, [0, 1, 2], n_layers=layers)
    if status:
        refuses(status, fcg.fcg_evict, c, [0], [0], [2], None)
        assert fcg.fcg_cache_export_layout(c, 0, 0)[1] == 3
    else:
        fcg.fcg_evict(c, [0], [0], [2], None)
        assert fcg.fcg_cache_export_layout(c, 0, layers - 1)[1] == 2


@pytest.mark.parametrize("page", [0, 16])
def test_a_prefix_squeezed_beside_itself_serves_others(page):
    """Sequences that run over a prefix go on with it; others start over its squeezed copy.  One with positions behind a
    prefix is no whole sequence and is refused, and so are those left by a prefix that was squeezed in place."""
    c = fcg.Cache(fcg.model_desc(2, 4, 2, 64, 1e4, "bf16"), 4, 200, page, 40 if page else 0, fcg.FCG_LAYOUT_ONLY)
    fcg.fcg_append(c, 0, [0] * 100, range(100), n_layers=2)
    fcg.fcg_append(c, 0, [1] * 40, range(100, 140), n_layers=2)

    def attend(pre, P, s, p):
        i = np.array([s, p], dtype=np.int32)
        fcg._check(fcg._L.fcg_prefix_attend(c.h, 0, pre, P, 1, fcg._p(i[:1]), fcg._p(i[1:]), None, None, None, None))

    attend(0, 100, 1, 139)
    evict(c, src=[0], dst=[2], keep=[50])
    attend(0, 100, 1, 139)
    fcg.fcg_append(c, 0, [3], [50], n_layers=2)
    attend(2, 50, 3, 50)
    refuses(E.FCG_EHOLE, evict, c, src=[1], dst=[1], keep=[10])
    evict(c, src=[0], dst=[0], keep=[50])
    refuses(E.FCG_EHOLE, attend, 0, 100, 1, 139)
    refuses(E.FCG_EHOLE, attend, 0, 50, 1, 139)

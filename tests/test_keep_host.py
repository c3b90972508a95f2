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

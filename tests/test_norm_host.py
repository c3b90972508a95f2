"""Norms with a rotary turn without a GPU: refusals, workspace sizes, the gradient's formula against differences."""
import copy
import ctypes
import pickle

import numpy as np
import pytest
import torch

from normutil import grad64, norm64
from opsutil import freqs64, turn64
from paper_2606_13097_amd import fcg

E = fcg


def refuses(status, f, *a, **k):
    with pytest.raises(fcg.FcgError) as e:
        f(*a, **k)
    assert e.value.status == status, str(e.value)


def V(data=64, layer=0, token=256, head=64):
    return fcg.TensorView(data, layer, token, head)


def N(weight=64, layer=0, head=0, eps=1e-6, offset=0.0):
    return fcg.NormDesc(weight, layer, head, eps, offset)


BAD_NORMS = [N(layer=-1), N(head=-1), N(eps=0.0), N(eps=-1.0), N(eps=float("nan")), N(eps=1e-50), N(eps=float("inf")),
             N(offset=float("nan")), N(offset=float("inf")), N(offset=1e39)]


def ref(x):
    return None if x is None else ctypes.byref(x)


def apply(rope, dt=1, d=64, layers=1, n=2, pos=64, hq=4, nq=None, q=None, qo=None, hk=0, nk=None, k=None, ko=None):
    fcg._check(fcg._L.fcg_norm_rope_apply(None if rope is None else rope.h, dt, d, layers, n, pos, hq, ref(nq), ref(q),
                                          ref(qo), hk, ref(nk), ref(k), ref(ko), None))


def test_apply_refusals_reach_no_kernel():
    r = fcg.fcg_rope_create(64)
    ok = dict(rope=r, nq=N(), q=V(), qo=V(1 << 20))
    for bad in (dict(rope=None), dict(dt=2), dict(d=32), dict(d=256), dict(layers=-1), dict(layers=65536), dict(n=-1),
                dict(n=(1 << 30) + 1), dict(hq=-1), dict(hq=4097), dict(pos=None), dict(qo=None), dict(q=V(None)),
                dict(qo=V(None)), dict(q=V(token=-1)), dict(qo=V(head=-1)), dict(qo=V(1 << 20, token=0)),
                dict(qo=V(1 << 20, token=255)), dict(layers=2, qo=V(1 << 20, layer=0)), dict(qo=V(64, token=512)),
                dict(hk=-1), dict(hk=1, k=V()), dict(rope=fcg.fcg_rope_create(128))):
        refuses(E.FCG_EINVAL, apply, **{**ok, **bad})
    for n in BAD_NORMS:
        refuses(E.FCG_EINVAL, apply, **{**ok, "nq": n})
        refuses(E.FCG_EINVAL, apply, **{**ok, "nk": n})
    for none in (dict(n=0), dict(layers=0), dict(hq=0), dict(q=None, qo=None)):
        apply(**{**ok, **none})


def side(heads=4, norm=None, x=None, grad=None, dx=None, dw=None):
    return fcg.NormSide(heads, None if norm is None else ctypes.pointer(norm), x or V(64), grad or V(1 << 16),
                        dx or V(1 << 20), dw)


def backward(rope, dt=1, d=64, layers=1, n=2, pos=64, q=None, k=None, ws=None, size=0):
    fcg._check(fcg._L.fcg_norm_rope_backward(None if rope is None else rope.h, dt, d, layers, n, pos, ref(q), ref(k), ws,
                                             size, None))


def test_backward_refusals_reach_no_kernel():
    r = fcg.fcg_rope_create(64)
    need = fcg.fcg_norm_rope_workspace(1, 2, 4, 0, 64)
    ok = dict(rope=r, q=side(norm=N(), dw=1 << 21), ws=1 << 22, size=need)
    none = V(None)
    for bad in (dict(rope=None), dict(dt=7), dict(d=96), dict(layers=65536), dict(n=-1), dict(pos=None), dict(ws=None),
                dict(ws=(1 << 22) + 8), dict(size=255), dict(q=side(-1)), dict(q=side(4097)), dict(k=side(-1)),
                dict(q=side(norm=N(weight=None), dw=64)), dict(q=side(dw=64)), dict(q=side(norm=N(), x=none)),
                dict(q=side(norm=N(), grad=none)), dict(q=side(norm=N(), dx=none)), dict(q=side(dx=V(64, token=1))),
                dict(q=side(norm=N(), dx=V(64, token=512))), dict(q=side(norm=N(), dx=V(1 << 16, token=512))),
                dict(q=side(norm=N(), grad=V(64, head=-4)))):
        refuses(E.FCG_EINVAL, backward, **{**ok, **bad})
    for n in BAD_NORMS:
        refuses(E.FCG_EINVAL, backward, **{**ok, "q": side(norm=n)})
    backward(r)
    backward(r, q=side(0), k=side(0))
    backward(r, layers=0, q=side(norm=N(), dw=64))
    backward(r, n=0, pos=None, q=side(norm=N()))      # no rows and no weights to clear


def test_workspace_holds_every_partial():
    for L, n, hq, hk, d in ((1, 1, 1, 0, 64), (1, 4407, 32, 8, 128), (48, 2000, 64, 8, 128), (3, 33, 0, 5, 64),
                            (1, 1 << 30, 4096, 4096, 128)):
        got = fcg.fcg_norm_rope_workspace(L, n, hq, hk, d)
        assert got % (4 * d) == 0 and got >= 4 * d * L * (hq + hk)
        assert got <= 4 * d * max(L * (hq + hk), 1024 * 9 + L * (hq + hk))
    assert fcg.fcg_norm_rope_workspace(0, 5, 4, 4, 64) == 0
    for bad in ((-1, 1, 1, 1, 64), (1, -1, 1, 1, 64), (1, 1, -1, 1, 64), (1, 1, 1, 4097, 64), (1, 1, 1, 1, 32)):
        refuses(E.FCG_EINVAL, fcg.fcg_norm_rope_workspace, *bad)
    assert fcg._L.fcg_norm_rope_workspace(64, 1, 1, 1, 1, None) == E.FCG_EINVAL


def test_append_norm_refusals_change_nothing():
    c = fcg.Cache(fcg.model_desc(1, 4, 2, 64, 1e4, "bf16"), 1, 32, flags=fcg.FCG_LAYOUT_ONLY)
    i = np.array([0], dtype=np.int32)

    def call(nq=None, nk=None, q=None, k=None, v=None):
        fcg._check(fcg._L.fcg_append_norm(c.h, 0, 1, 1, fcg._p(i), fcg._p(i), None, ref(nq), ref(nk), ref(q), ref(q), ref(k),
                                          ref(v), 0, None))

    refuses(E.FCG_EINVAL, call, nk=N())
    refuses(E.FCG_EINVAL, call, nq=N())
    for n in BAD_NORMS:
        refuses(E.FCG_EINVAL, call, nk=n, k=V(), v=V())
    refuses(E.FCG_EINVAL, call, nk=N(), k=V(), v=V())         # a layout-only cache takes no data
    assert fcg.fcg_cache_export_layout(c, 0, 0)[1] == 0
    call()                                                    # a reservation, as fcg_append makes it
    assert fcg.fcg_cache_export_layout(c, 0, 0)[1] == 1
    assert fcg._L.fcg_append_norm(None, 0, 0, 0, None, None, None, None, None, None, None, None, None, 0, None) == E.FCG_EINVAL


def test_norm_weights_in_the_binding():
    w = torch.zeros(3, 4, 64)
    assert (fcg.Norm(w).desc.layer, fcg.Norm(w).desc.head) == (256, 64)
    assert (fcg.Norm(w[:, :1]).desc.layer, fcg.Norm(w[:, :1]).desc.head) == (256, 0)
    assert (fcg.Norm(w[0]).desc.layer, fcg.Norm(w[0]).desc.head) == (0, 64)
    assert (fcg.Norm(w[0, 0]).desc.layer, fcg.Norm(w[0, 0]).desc.head) == (0, 0)
    assert fcg.Norm(None).desc.weight is None
    assert fcg.Norm(w).dweight_shape(3, 4) == (3, 4, 64) and fcg.Norm(w[0, 0]).dweight_shape(3, 4) == (3, 1, 64)
    for bad in (torch.zeros(2, 2, 2, 64), torch.zeros(64, 64).T[:, :5], torch.zeros(())):
        with pytest.raises(ValueError):
            fcg.Norm(bad)
    with pytest.raises(ValueError):
        fcg.fcg_norm_rope_apply(fcg.fcg_rope_create(64), torch.zeros(1, dtype=torch.int32), torch.zeros(1, 1, 64))


def test_gradient_formula_against_differences():
    """The reference of the GPU tests: autograd of the definition, against central differences in 64 bits."""
    g = torch.Generator().manual_seed(3)
    x, gy = (torch.randn(1, 2, 2, 16, generator=g, dtype=torch.float64) for _ in range(2))
    w = torch.randn(1, 1, 2, 16, generator=g, dtype=torch.float64)
    f, pos, eps, m = freqs64(16, 1e4), [5, 70000], 1e-3, 1.5
    dx, dw = grad64(x, w, gy, eps, pos, f, True, m)

    def loss(x, w):
        return float((turn64(norm64(x, w, eps), pos, f, True, m) * gy).sum())

    h = 1e-6
    for i in range(0, x.numel(), 5):
        e = torch.zeros_like(x).view(-1)
        e[i] = h
        e = e.view(x.shape)
        assert abs((loss(x + e, w) - loss(x - e, w)) / (2 * h) - float(dx.view(-1)[i])) < 1e-7
    for i in range(w.numel()):
        e = torch.zeros_like(w).view(-1)
        e[i] = h
        e = e.view(w.shape)
        assert abs((loss(x, w + e) - loss(x, w - e)) / (2 * h) - float(dw.sum(1, keepdim=True).view(-1)[i])) < 1e-7


def test_a_norm_goes_by_the_weights_of_the_call():
    """A parameter's storage moves under it (Module.to, an optimiser's swap): address and strides are the present ones."""
    w = torch.nn.Parameter(torch.zeros(4, 64), requires_grad=False)
    norm = fcg.Norm(w, eps=1e-5, offset=1.0)
    old = w.data                                  # keeps the first storage, so that no other takes its address
    w.data = torch.ones(4, 128)[:, 64:]
    assert norm.desc.weight == w.data_ptr() != old.data_ptr() and (norm.desc.layer, norm.desc.head) == (0, 128)
    desc = fcg._norm_ref(norm, 1, 4, 64, torch.float32, w.get_device(), "q_norm")._obj
    assert (desc.weight, desc.layer, desc.head, desc.eps, desc.offset) == (w.data_ptr(), 0, 128, 1e-5, 1.0)
    x = torch.zeros(2, 4, 64)
    side = fcg._norm_side(x, norm, x, x.clone(), None, (1, 2, 4, 64), torch.float32, w.get_device(), "q")
    assert (side.norm.contents.weight, side.norm.contents.head) == (w.data_ptr(), 128)
    w.data = torch.ones(4, 64)[:1]
    assert norm.desc.head == 0 and norm.dweight_shape(2, 4) == (2, 1, 64)
    w.data = torch.zeros(64, 4).T
    with pytest.raises(ValueError):               # elements of a head that are no longer adjacent
        fcg._norm_ref(norm, 1, 4, 64, torch.float32, w.get_device(), "q_norm")


def test_append_norm_of_no_tokens_is_no_error():
    """As fcg_append of none: an empty tensor has no address."""
    c = fcg.Cache(fcg.model_desc(2, 4, 2, 64, 1e4, "bf16"), 1, 32, flags=fcg.FCG_LAYOUT_ONLY)
    none = np.zeros(0, dtype=np.int32)
    for layers, n in ((1, 0), (2, 0), (0, 0), (0, 1)):
        i = np.zeros(n, dtype=np.int32)
        for q, k in ((None, None), (V(None), V(None))):
            args = (c.h, 0, layers, n, fcg._p(i), fcg._p(i), None)
            fcg._check(fcg._L.fcg_append_norm(*args, ref(N()), ref(N()), ref(q), ref(q), ref(k), ref(k), 0, None))
    assert fcg.fcg_cache_export_layout(c, 0, 0)[1] == 0
    refuses(E.FCG_EINVAL, lambda: fcg._check(fcg._L.fcg_append_norm(
        c.h, 0, 1, 0, fcg._p(none), fcg._p(none), None, ref(N(eps=0.0)), None, None, None, None, None, 0, None)))


def test_copies_of_a_norm_stand_alone():
    """A model that holds norms can be copied; a copy with other weights leaves the first one's description as it is."""
    norm = fcg.Norm(torch.zeros(4, 64), 1e-5, 1.0)
    for twin in (copy.copy(norm), copy.deepcopy(norm), pickle.loads(pickle.dumps(norm))):
        first = fcg._norm_ref(norm, 1, 4, 64, torch.float32, -1, "q")._obj
        twin.weight = torch.ones(4, 128)[:, :64]
        other = fcg._norm_ref(twin, 1, 4, 64, torch.float32, -1, "q")._obj
        assert (first.weight, first.head) == (norm.weight.data_ptr(), 64)
        assert (other.weight, other.head, other.eps, other.offset) == (twin.weight.data_ptr(), 128, 1e-5, 1.0)

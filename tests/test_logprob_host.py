"""Log probabilities without a GPU: refusals, workspace sizes, checks of the binding."""
import numpy as np
import pytest
import torch

from paper_2606_13097_amd import fcg

E = fcg


def refuses(status, f, *a, **k):
    with pytest.raises(fcg.FcgError) as e:
        f(*a, **k)
    assert e.value.status == status, str(e.value)


def forward(dt=1, n=2, vocab=100, x=64, stride=100, targets=64, lp=64, ent=64, lse=64, k=4, ids=64, tlp=64, ws=64, size=1 << 20):
    fcg._check(fcg._L.fcg_token_logprobs(dt, n, vocab, x, stride, targets, lp, ent, lse, k, ids, tlp, ws, size, None))


def test_forward_refusals_reach_no_kernel():
    big = dict(vocab=100000, stride=100000)
    need = fcg.fcg_token_logprobs_workspace(2, 100000, 4)
    assert need > 0
    for bad in (dict(dt=2), dict(dt=-1), dict(n=-1), dict(vocab=0), dict(vocab=(1 << 30) + 1), dict(stride=-1), dict(k=-1),
                dict(k=65), dict(vocab=3), dict(x=None), dict(targets=None), dict(ids=None), dict(ws=None, **big),
                dict(ws=72, **big), dict(size=need - 1, **big)):
        refuses(E.FCG_EINVAL, forward, **bad)
    forward(n=0, x=None)
    forward(lp=None, ent=None, lse=None, k=0)          # nothing asked for


def backward(dt=1, n=2, vocab=100, x=64, stride=100, targets=64, lse=64, ent=64, gl=64, gh=64, gs=64, dx=1 << 20, ds=100):
    fcg._check(fcg._L.fcg_token_logprobs_backward(dt, n, vocab, x, stride, targets, lse, ent, gl, gh, gs, dx, ds, None))


def test_backward_refusals_reach_no_kernel():
    for bad in (dict(dt=2), dict(n=-1), dict(vocab=0), dict(stride=-1), dict(x=None), dict(lse=None), dict(dx=None),
                dict(targets=None), dict(ent=None), dict(ds=99), dict(dx=64, ds=101)):
        refuses(E.FCG_EINVAL, backward, **bad)
    backward(n=0, x=None)


def test_workspace():
    w = fcg.fcg_token_logprobs_workspace
    assert w(0, 1000) == 0 and w(1, 4096, 64) == 0 and w(1024, 200000, 64) == 0
    assert w(1, 131072, 20) == 32 * (16 + 8 * 20)
    for n in (1, 3, 100, 1023):
        for vocab in (8193, 50021, 1 << 30):
            for k in (0, 64):
                assert 0 < w(n, vocab, k) <= n * 32 * (16 + 8 * k)
    for bad in ((-1, 10, 0), (1, 0, 0), (1, (1 << 30) + 1, 0), (1, 10, -1), (1, 100, 65)):
        refuses(E.FCG_EINVAL, w, *bad)
    assert fcg._L.fcg_token_logprobs_workspace(1, 1, 0, None) == E.FCG_EINVAL


def test_measure_refusals():
    loc = fcg.Locality(3)
    i = np.array([0, 1], dtype=np.int32)

    def call(h=loc.h, n=2, funcs=(0, 1), lens=(1, 1), lp=64):
        f, m = np.array(funcs, dtype=np.int32), np.array(lens, dtype=np.int32)
        fcg._check(fcg._L.fcg_locality_measure_ppl(h, n, fcg._p(f), fcg._p(m), lp, None))

    refuses(E.FCG_EINVAL, call, h=None)
    refuses(E.FCG_EINVAL, call, n=-1)
    refuses(E.FCG_EINVAL, call, lp=None)
    refuses(E.FCG_EINVAL, call, lens=(1, 0))
    refuses(E.FCG_ERANGE, call, funcs=(0, 3))
    refuses(E.FCG_ERANGE, call, funcs=(-1, 0))
    call(n=0)
    assert not fcg.fcg_locality_scores(loc).any()


def test_checks_of_the_binding():
    x = torch.zeros(2, 10)
    with pytest.raises(ValueError):
        fcg.fcg_token_logprobs(x)
    with pytest.raises(ValueError):
        fcg.fcg_token_logprobs(x.requires_grad_())
    with pytest.raises(ValueError):
        fcg.fcg_locality_measure_ppl(fcg.Locality(2), [0], [1], torch.zeros(1))

"""The bounds of the prefix-attention tests reject results that are wrong in small ways: mistakes planted in the oracle."""
import math

import numpy as np
import pytest
import torch

from opsbounds import NORM_LIMIT, check_attend_tight
from opsutil import attend64, freqs64, turn64


def bf(x):
    return x.to(torch.bfloat16)


def rejects(*a, **k):
    with pytest.raises(AssertionError, match="bound|norm|lse"):
        check_attend_tight(*a, **k)


@pytest.mark.parametrize("own", [1, 20, 33])
def test_bound_rejects_wrong_own_keys(own):
    """The shapes of the joined test: 241 shared keys, a few own ones."""
    g = torch.Generator().manual_seed(own)
    P, hq, hkv, d = 241, 8, 2, 64
    w = freqs64(32, 1e4, "parts", 4.0, 32768.0)
    raw = torch.randn((P + own, hkv, d), generator=g)
    K, V = bf(turn64(bf(raw), np.arange(P + own), w, True, 1.1)), bf(torch.randn((P + own, hkv, d), generator=g))
    q = bf(torch.randn((1, hq, d), generator=g))
    pos = [P + own - 1]
    ref = attend64(q, K, V, pos, P)
    check_attend_tight(bf(ref[0]), ref[1].float(), ref, "bf16", P + own, d, "right")
    K2 = K.clone()
    K2[P:] = bf(raw[P:])                              # own keys not encoded
    V2 = V.clone()
    V2[-1] = V[-2]                                    # the newest value row of its neighbour
    for what, k, v, p in (("no own keys", K[:P], V[:P], P - 1), ("not the newest key", K[:-1], V[:-1], P + own - 2),
                          ("own keys as they came", K2, V, P + own - 1), ("a value row of its neighbour", K, V2, P + own - 1)):
        o, lse, _, _ = attend64(q, k, v, [p], P)
        rejects(bf(o), None, ref, "bf16", P + own, d, what)
        if what != "a value row of its neighbour":
            rejects(bf(ref[0]), lse.float(), ref, "bf16", P + own, d, what)


def test_norm_bound_tells_partials_apart():
    """The kernels' roundings over a long split prefix, on the host: fp16 partials pass, bf16 ones do not."""
    g = torch.Generator().manual_seed(1)
    n, d, rows, split = 4321, 128, 64, 320
    K, V, q = (bf(torch.randn(s, generator=g)).double() for s in ((n, d), (n, d), (rows, d)))
    z = (q @ K.T) / math.sqrt(d)
    m = z.amax(-1, keepdim=True)
    p = torch.exp(z - m)
    out, l = torch.softmax(z, -1) @ V, p.sum(-1, keepdim=True)
    for kind, lo, hi in (("f32", 2.1e-3, NORM_LIMIT), ("f16", 2.1e-3, NORM_LIMIT), ("bf16", 2.6e-3, 3e-3)):
        o = torch.zeros_like(out)
        for k0 in range(0, n, split):
            part = bf(p[:, k0:k0 + split]).double() @ V[k0:k0 + split]
            if kind == "f16":
                up = 2.0 ** (15 - torch.frexp(part.abs().amax(-1, keepdim=True))[1].double())
                part = (part * up).half().double() / up
            elif kind == "bf16":
                part = bf(part).double()
            o += part
        rel = float((bf(o / l).double() - out).norm() / out.norm())
        assert lo <= rel <= hi, (kind, rel)

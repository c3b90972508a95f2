"""Rotary handles, append and prefix attention without a GPU: calls at the edges of what their documentation allows."""
import numpy as np
import pytest
import torch

from paper_2606_13097_amd import fcg


def refuses(status, f, *a, **k):
    with pytest.raises(fcg.FcgError) as e:
        f(*a, **k)
    assert e.value.status == status, str(e.value)


def test_rope_values_that_the_kernels_cannot_hold_are_refused():
    """The factor goes to the kernels in fp32, where 1e-50 is 0 and 1e39 infinite; the angle p w of a frequency of 1e300
    is infinite at far positions, and its cos no number."""
    for m in (1e-50, 1e-39, 1e39, 1e300, -1.0):
        refuses(fcg.FCG_EINVAL, fcg.fcg_rope_create, 64, attn_factor=m)
    for m in (2.0 ** -126, 3e38):
        fcg.fcg_rope_create(64, attn_factor=m)
    w = np.zeros(32)
    for f in (1e300, -1e300, float("nan"), float("inf")):
        w[31] = f
        refuses(fcg.FCG_EINVAL, fcg.fcg_rope_create, 64, scaling=fcg.FCG_ROPE_GIVEN, freqs=w)
    w[31] = -3e298
    assert np.array_equal(fcg.fcg_rope_frequencies(fcg.fcg_rope_create(64, scaling=fcg.FCG_ROPE_GIVEN, freqs=w)), w)


def test_angle_error_of_a_pair():
    """The bound that fcg.h gives, on the host in the kernel's steps (float64 turns, their product's distance to a whole
    turn) against 80-bit products: every pair of some forms, positions over all of int32."""
    ld = np.longdouble
    assert np.finfo(ld).nmant >= 63
    two_pi = ld(2) * ld("3.14159265358979323846264338327950288")
    p = np.unique(np.r_[np.random.default_rng(1).integers(-2 ** 31, 2 ** 31, 2000), -2 ** 31, 2 ** 31 - 1, 1, 2 ** 24 + 1])
    for theta in (1e4, 1e6):
        w = theta ** (-2.0 * np.arange(64) / 128)
        t = p[:, None].astype(np.float64) * (w / 6.283185307179586477)
        got = (t - np.rint(t)).astype(ld)
        exact = p[:, None].astype(ld) * w.astype(ld)
        off = got - exact / two_pi
        off = np.abs(off - np.rint(off)) * two_pi
        assert (off <= 2.0 ** -51 * np.abs(exact) + 1e-18).all()
        assert (off > 2.0 ** -54 * np.abs(exact)).any()        # (and not far below it)


def test_tensors_that_need_a_gradient_are_refused():
    """The calls record none: a result without one, silently, would train nothing."""
    x = torch.zeros((2, 4, 64), requires_grad=True)
    with pytest.raises(ValueError, match="gradient"):
        fcg._view(x, (1, 2, 4, 64), torch.float32, None, "q")
    for t in (x.detach(), x):
        with torch.no_grad(), pytest.raises(ValueError, match="GPU"):     # past that check
            fcg._view(t, (1, 2, 4, 64), torch.float32, None, "q")


def test_calls_take_the_stream_of_their_caches_device(monkeypatch):
    """Without a stream: torch's current one of the cache's device, not of the current device."""
    d = fcg.model_desc(1, 4, 2, 64, 1e4, "bf16")
    c = fcg.Cache(d, 2, 64, 16, 8, flags=fcg.FCG_LAYOUT_ONLY)
    lib = fcg.Library(d, 64, 1, flags=fcg.FCG_LAYOUT_ONLY)
    fcg.fcg_lib_add_segment(lib, 16, 0)
    rope = fcg.fcg_rope_create(32)
    seen = {}
    for name in ("fcg_graft_rope", "fcg_append", "fcg_prefix_attend"):
        monkeypatch.setattr(fcg._L, name, lambda *a, name=name: seen.setdefault(name, a[-1]) and 0)
    monkeypatch.setattr(fcg, "_raw_stream", lambda device: 1000 + device)
    monkeypatch.setattr(fcg, "_current_stream", lambda: 1)
    c.device = 5
    fcg.fcg_graft_rope(c, lib, rope, [0], [0], [0])
    fcg.fcg_append(c, 0, [0], [20])
    fcg.fcg_prefix_attend(c, 0, 0, 16, [0], [15], None, None)
    assert seen == dict.fromkeys(seen, 1005) and len(seen) == 3


def test_append_refuses_a_layer_count_that_its_keys_contradict():
    """n_layers is that of reservations; keys bring theirs.  Another one was ignored: the other layers stayed unwritten."""
    c = fcg.Cache(fcg.model_desc(4, 4, 2, 64, 1e4, "bf16"), 2, 64, flags=fcg.FCG_LAYOUT_ONLY)
    for shape, n in (((3, 2, 64), 2), ((2, 3, 2, 64), 3), ((2, 3, 2, 64), 4), ((1, 3, 2, 64), 2)):
        with pytest.raises(ValueError, match="layers"):
            x = torch.zeros(shape, dtype=torch.bfloat16)
            fcg.fcg_append(c, 0, [0, 0, 0], [0, 1, 2], x, x, n_layers=n)
    for shape, n in (((3, 2, 64), 1), ((2, 3, 2, 64), 1), ((2, 3, 2, 64), 2)):      # past that check
        with pytest.raises(ValueError, match="GPU"):
            x = torch.zeros(shape, dtype=torch.bfloat16)
            fcg.fcg_append(c, 0, [0, 0, 0], [0, 1, 2], x, x, n_layers=n)

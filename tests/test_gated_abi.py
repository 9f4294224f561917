"""Entry points of the root-mean-square norm and the gated layer without a GPU: NULL arguments are errors, not crashes; and what the
plain statements in gated_plain.py promise (they are what the GPU tests compare with)."""
import ctypes
import os

import numpy as np
import pytest

import gated_plain as plain

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2105_13336_amd", "libtensile.so")


def test_null_arguments_are_errors():
    if not os.path.exists(LIB):
        from paper_2105_13336_amd.build import build_library
        build_library()
    lib = ctypes.CDLL(LIB)
    lib.tensile_last_error.restype = ctypes.c_char_p
    p = None
    calls = {"rms_norm": (p, p, p, p, 0, ctypes.c_double(1e-6), p, p, p, p, p), "rms_norm_backward": (p, p, p, p, p, 0, p, p, p, p),
             "gated_linear": (p, p, p, p, p, p, 0, 0, p, p, p, p), "gated_linear_backward": (p, p, p, p, 0, p, p, p, p, p, p, p)}
    for name, args in calls.items():
        assert getattr(lib, "tensile_" + name)(*args) == -1
        assert name.encode() in lib.tensile_last_error() and b"NULL" in lib.tensile_last_error()


def test_an_unknown_activation_is_refused_before_any_call():
    import paper_2105_13336_amd as P
    with pytest.raises(P.TensileError) as e:
        P.binding._activation("relu6")
    assert e.value.code == -1 and "relu6" in str(e.value)


def test_plain_backward_passes_are_derivatives():
    rng = np.random.default_rng(12)
    h = 1e-6
    s, gamma, dy = rng.standard_normal((3, 20)), rng.standard_normal(20), rng.standard_normal((3, 20))
    _, xhat, rstd = plain.rms_norm(s, gamma, 0.1)
    dx, dgamma = plain.rms_norm_backward(dy, xhat, rstd, gamma)
    loss = lambda s, g: (dy * plain.rms_norm(s, g, 0.1)[0]).sum()
    d, e = rng.standard_normal(s.shape), rng.standard_normal(20)
    assert abs((loss(s + h * d, gamma) - loss(s - h * d, gamma)) / (2 * h) - np.vdot(dx, d)) < 1e-6
    assert abs((loss(s, gamma + h * e) - loss(s, gamma - h * e)) / (2 * h) - np.vdot(dgamma, e)) < 1e-6
    x = np.linspace(-8, 8, 161)
    for act in plain.ACTS:
        slope = plain.activation(x, act)[1]
        assert np.abs((plain.activation(x + h, act)[0] - plain.activation(x - h, act)[0]) / (2 * h) - slope).max() < 1e-8
        x0, wg, wu, bg, bu = (rng.standard_normal(n) for n in ((4, 6), (5, 6), (5, 6), 5, 5))
        dh = rng.standard_normal((4, 5))
        value, g, u = plain.gated(x0, wg, wu, bg, bu, act)
        dgate, dup, again = plain.gated_grad(dh, g, u, act)
        assert np.array_equal(again, value)
        loss = lambda x: (dh * plain.gated(x, wg, wu, bg, bu, act)[0]).sum()
        d = rng.standard_normal(x0.shape)
        assert abs((loss(x0 + h * d) - loss(x0 - h * d)) / (2 * h) - np.vdot(dgate @ wg + dup @ wu, d)) < 1e-6

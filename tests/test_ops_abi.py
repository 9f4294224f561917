"""The operators' entry points without a GPU: NULL arguments are errors, not crashes; and what the plain statements in
ops_plain.py promise (they are what the GPU tests compare with)."""
import ctypes
import os

import numpy as np
import pytest

import ops_plain as plain

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2105_13336_amd", "libtensile.so")


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(LIB):
        from paper_2105_13336_amd.build import build_library
        build_library()
    lib = ctypes.CDLL(LIB)
    lib.tensile_last_error.restype = ctypes.c_char_p
    return lib


def test_null_arguments_are_errors(lib):
    p = None
    calls = {"ckpt_pack": (p,) * 4, "ckpt_unpack": (p,) * 4,
             "layer_norm": (p, p, p, p, p, 0, ctypes.c_double(1e-5), p, p, p, p, p),
             "layer_norm_backward": (p, p, p, p, p, 0, p, p, p, p, p),
             "gelu": (p, p, p, p, 0, p), "gelu_backward": (p, p, p, p, p, 0, p),
             "linear_grad": (p, p, p, p, p, 0, p, p, p)}
    for name, args in calls.items():
        assert getattr(lib, "tensile_" + name)(*args) == -1
        assert name.encode() in lib.tensile_last_error() and b"NULL" in lib.tensile_last_error()
    assert lib.tensile_ops_create(None) == -1 and b"NULL" in lib.tensile_last_error()
    lib.tensile_ops_free.restype = None
    lib.tensile_ops_free(None)     # allowed


def test_checkpoints_live_on_the_gpu():
    import torch

    import paper_2105_13336_amd as P
    with pytest.raises(P.TensileError) as e:
        P.Checkpoint(torch.zeros(2, 32, dtype=torch.int8), torch.zeros(2, 1, dtype=torch.uint8))
    assert e.value.code == -1


@pytest.mark.parametrize("cap", [136, 248])
def test_plain_packing(cap):
    """Half a scale is the most a value is off, the scale is the smallest that does, and a second packing changes nothing."""
    rng = np.random.default_rng(cap)
    x = rng.standard_normal((64, 77)) * np.exp2(rng.integers(-20, 9, (64, 1)))
    q, code = plain.pack(x, cap)
    value = plain.unpack(q, code)
    scale = np.repeat(np.exp2(code.astype(float) - 127), 32, axis=1)[:, :77]
    assert (np.abs(value - x) <= scale / 2).all() and (np.abs(q.astype(int)) <= 127).all()
    assert (np.abs(plain.groups_of(q.astype(float))).max(axis=2)[code > 1] >= 63.5).all()
    q2, code2 = plain.pack(value, cap)
    assert np.array_equal(plain.unpack(q2, code2), value)


def test_plain_backward_passes_are_derivatives():
    rng = np.random.default_rng(11)
    s, gamma, beta, dy = rng.standard_normal((3, 20)), rng.standard_normal(20), rng.standard_normal(20), rng.standard_normal((3, 20))
    _, xhat, rstd = plain.layer_norm(s, gamma, beta, 0.1)
    dx, dgamma, dbeta = plain.layer_norm_backward(dy, xhat, rstd, gamma)
    loss = lambda s, g, b: (dy * plain.layer_norm(s, g, b, 0.1)[0]).sum()
    h = 1e-6
    for got, which in ((dx, 0), (dgamma, 1), (dbeta, 2)):
        d = rng.standard_normal(got.shape)
        args = [s, gamma, beta]
        plus, minus = list(args), list(args)
        plus[which], minus[which] = args[which] + h * d, args[which] - h * d
        assert abs((loss(*plus) - loss(*minus)) / (2 * h) - np.vdot(got, d)) < 1e-6
    x = np.linspace(-6, 6, 101)
    for tanh in (False, True):
        y, slope = plain.gelu(x, tanh)
        assert np.abs((plain.gelu(x + h, tanh)[0] - plain.gelu(x - h, tanh)[0]) / (2 * h) - slope).max() < 1e-8

"""The root-mean-square norm and the gated layer, plainly and in 64 bits (numpy), and how far 32-bit arithmetic may be from that."""
from __future__ import annotations

import numpy as np

from ops_plain import U, gelu

ACTS = ["silu", "gelu", "gelu_tanh"]


def rms_norm(s, gamma, eps):
    """-> (y, xhat, rstd)"""
    rstd = 1 / np.sqrt((s * s).mean(axis=1) + eps)
    xhat = s * rstd[:, None]
    return xhat * gamma, xhat, rstd


def rms_norm_backward(dy, xhat, rstd, gamma):
    """-> (dx, dgamma)"""
    t = dy * gamma
    return rstd[:, None] * (t - xhat * (t * xhat).mean(axis=1, keepdims=True)), (dy * xhat).sum(axis=0)


def activation(x, act):
    """-> (value, derivative)"""
    if act == "gelu":
        return gelu(x, False)
    # x times the logistic function of z, of which (1 + tanh(z/2))/2 is another form (one that is 0 in 64 bits from z = -37 on)
    k, a = np.sqrt(2 / np.pi), 0.044715
    z, dz = (x, 1.0) if act == "silu" else (2 * k * (x + a * x ** 3), 2 * k * (1 + 3 * a * x * x))
    e = np.exp(-np.abs(z))
    p, rest = np.where(z < 0, e, 1.0) / (1 + e), np.where(z < 0, 1.0, e) / (1 + e)
    with np.errstate(invalid="ignore", over="ignore"):
        return x * p, p + np.where(e == 0, 0.0, x * p * rest * dz)


def activation_error(x, act, dtype):
    """How far value and derivative may be off.  SiLU: its exponential's argument is rounded (|x|/2 units, and 1.5 of the function and the
    reciprocal each), then three products; GELU as tensile.h has it.  A value below 2^-126 is no normal number of 32 bits (GELU of -15 is 5e-50): it
    may be 0 there, which is off by 2^-126 at most; and tensile.h's bound ends at -10, where GELU is -7.6e-23, from where on it falls to 0."""
    value, slope = activation(x, act)
    least = np.where((x < -10) & (act != "silu"), 7.7e-23, 2.0 ** -126)
    if act == "silu":
        unit = U * (8 + 2 * np.abs(x))
        return unit * np.abs(value) + least, unit * (1 + np.abs(x)) + least
    if dtype == "f32":
        return U * (16 + 15 * np.abs(x) + 2 * x * x) * np.abs(value) + least, 5e-7 + 0 * x
    return 5e-7 * np.abs(x), 1e-6 * (1 + np.abs(x))


def gated(x, wg, wu, bg, bu, act):
    """-> (h, g, u)"""
    g, u = x @ wg.T + bg, x @ wu.T + bu
    return activation(g, act)[0] * u, g, u


def gated_grad(dh, g, u, act):
    """-> (dgate, dup, h)"""
    value, slope = activation(g, act)
    return dh * u * slope, dh * value, value * u


def chain(terms, dtype, parts=1):
    """Additions that a term of a sum of so many may pass through: a matrix instruction adds 16 products (2 in 32 bits) to a sum, in
    whatever order; the parts of a sum that is split are added up behind."""
    return terms / (2 if dtype == "f32" else 16) + (2 if dtype == "f32" else 16) + parts + 8

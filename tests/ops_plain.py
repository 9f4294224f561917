"""The operators on 8-bit checkpoints, plainly and in 64 bits (numpy), and how far 32-bit arithmetic may be from that.

``U`` is the unit of 32-bit sums (2^-24); a bound of the form ``c * U * (sum of magnitudes)`` holds for any order of a sum in
which no addend passes through more than c additions.
"""
from __future__ import annotations

import math

import numpy as np

U = 2.0 ** -24
GROUP = 32
#: half a unit in the last place, relative: 2^-p for a type of p significant bits (24, 8 and 11, the leading one counted)
ROUND = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
#: half the distance between the smallest numbers of the type
FLOOR = {"f32": 0.0, "bf16": 0.0, "f16": 2.0 ** -25}
CAP = {"f32": 248, "bf16": 248, "f16": 136}


def groups_of(x):
    rows, cols = x.shape
    g = np.zeros((rows, (cols + GROUP - 1) // GROUP * GROUP))
    g[:, :cols] = x
    return g.reshape(rows, -1, GROUP)


def code_of(a, cap):
    """Scale codes for the groups' largest magnitudes a (64 bits): smallest e with a / 2^e < 127.5, code e + 127 in [1, cap]."""
    code = np.full(a.shape, 255, dtype=np.int64)
    fine = np.isfinite(a)
    mant, expo = np.frexp(np.where(fine, a, 1.0))              # a = mant * 2^expo, 0.5 <= mant < 1
    e = expo - 7 + (mant >= 127.5 / 128)
    e = np.where(a == 0, -1000, e)
    code[fine] = np.clip(e + 127, 1, cap)[fine]
    return code


def pack(x, cap):
    """-> (q int8, codes) of x"""
    rows, cols = x.shape
    g = groups_of(x)
    code = code_of(np.abs(g).max(axis=2), cap)
    e = np.where(code == 255, 0, code - 127)
    with np.errstate(invalid="ignore", over="ignore"):
        q = np.clip(np.rint(g / np.exp2(e.astype(np.float64))[:, :, None]), -127, 127)
    q = np.where((code == 255)[:, :, None], 0, q)
    return q.reshape(rows, -1)[:, :cols].astype(np.int8), code.astype(np.uint8)


def unpack(q, code):
    cols = q.shape[1]
    scale = np.where(code == 255, np.nan, np.where(code == 0, 0.0, np.exp2(code.astype(np.float64) - 127)))
    return q.astype(np.float64) * np.repeat(scale, GROUP, axis=1)[:, :cols]


def layer_norm(s, gamma, beta, eps):
    """-> (y, xhat, rstd)"""
    mean = s.mean(axis=1, keepdims=True)
    rstd = 1 / np.sqrt(((s - mean) ** 2).mean(axis=1, keepdims=True) + eps)
    xhat = (s - mean) * rstd
    return xhat * gamma + beta, xhat, rstd[:, 0]


def layer_norm_backward(dy, xhat, rstd, gamma):
    """-> (dx, dgamma, dbeta)"""
    h = dy * gamma
    dx = rstd[:, None] * (h - h.mean(axis=1, keepdims=True) - xhat * (h * xhat).mean(axis=1, keepdims=True))
    return dx, (dy * xhat).sum(axis=0), dy.sum(axis=0)


def gelu(x, tanh):
    """-> (y, dy/dx)"""
    if tanh:
        k = math.sqrt(2 / math.pi)
        t = np.tanh(k * (x + 0.044715 * x ** 3))
        return 0.5 * x * (1 + t), 0.5 * (1 + t) + 0.5 * x * (1 - t * t) * k * (1 + 3 * 0.044715 * x * x)
    from scipy.special import erfc
    cdf = 0.5 * erfc(-x / math.sqrt(2))
    return x * cdf, cdf + x * np.exp(-0.5 * x * x) / math.sqrt(2 * math.pi)


def linear_grad(dy, X):
    """-> (dw, dbias)"""
    return dy.T @ X, dy.sum(axis=0)

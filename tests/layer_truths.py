"""Plain 64-bit forms of the layer operators and the error bounds that follow
from how the library computes them (numpy only, no code of the library)."""
from __future__ import annotations

import math

import numpy as np

ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")
UNIT = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}   # one rounding
TINY = {"float32": 2.0 ** -149, "bfloat16": 2.0 ** -133, "float16": 2.0 ** -24}   # spacing near zero
# An activation is evaluated in fp32 to within ACT |z|, its slope to within
# ACT (1 + |z|): a few fp32 roundings for float32, a sixteenth of the result's
# own rounding for the 16-bit types.
ACT = {"float32": 2.0 ** -20, "bfloat16": 2.0 ** -15, "float16": 2.0 ** -15}

_erfc = np.vectorize(math.erfc, otypes=[np.float64])


def phi(z):
    return 0.5 * _erfc(-z / math.sqrt(2.0)) if z.size else z


def value(z, act):
    if act == "relu":
        return np.where(z <= 0, 0.0, z)
    if act == "gelu":
        return z * phi(z)
    if act == "gelu_tanh":
        return 0.5 * z * (1 + np.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    if act == "silu":
        return z / (1 + np.exp(-z))
    return z


def slope(z, act):
    if act == "relu":
        return np.where(z <= 0, 0.0, 1.0)
    if act == "gelu":
        return phi(z) + z * np.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":
        a = math.sqrt(2 / math.pi)
        t = np.tanh(a * (z + 0.044715 * z ** 3))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * a * (1 + 3 * 0.044715 * z * z)
    if act == "silu":
        s = 1 / (1 + np.exp(-z))
        return s * (1 + z * (1 - s))
    return np.ones_like(z)


def linear(F, X, bias, act, residual):
    z = F @ X
    if bias is not None:
        z = z + bias[:, None]
    o = value(z, act)
    return (o if residual is None else o + residual), z


def linear_bound(F, X, bias, act, residual, dtype):
    """(bound of O, bound of Z): fp32 sums of ci products and the additions that
    follow (gamma), an activation whose slope is at most 1.13, one rounding."""
    o, z = linear(F, X, bias, act, residual)
    g = (F.shape[1] + 4) * 2.0 ** -24
    sums = np.abs(F) @ np.abs(X) + (0 if bias is None else np.abs(bias)[:, None])
    ez = 1.001 * g * sums
    eo = 1.13 * ez + (0 if act == "none" else ACT[dtype] * np.abs(z))
    if residual is not None:
        eo = eo + 2.0 ** -24 * (np.abs(o) + np.abs(residual))
    u = UNIT[dtype]
    return eo + u * (np.abs(o) + eo) + TINY[dtype], ez + u * (np.abs(z) + ez) + TINY[dtype]


def backward(F, X, dO, z, act):
    dz = dO if act == "none" else (np.where(z <= 0, 0.0, dO) if act == "relu" else dO * slope(z, act))
    return F.T @ dz, dz @ X.T, dz.sum(1), dz


def backward_bound(F, X, dO, z, act, dtype):
    """Bounds of dX, dF, dbias: dZ to the slope's accuracy and one rounding to
    the type (not for dbias, nor without an activation), fp32 sums, one rounding
    of each result."""
    dX, dF, db, dz = backward(F, X, dO, z, act)
    u = UNIT[dtype]
    es = np.zeros_like(dO) if act in ("none", "relu") else (ACT[dtype] * (1 + np.abs(z)) + 2.0 ** -24) * np.abs(dO)
    ez = es + (0 if act == "none" else u * (np.abs(dz) + es) + TINY[dtype])
    top = np.abs(dz) + ez
    g = 2.0 ** -24
    kn, ci, t = F.shape[0], F.shape[1], X.shape[1]
    eX = np.abs(F).T @ ez + 1.001 * (kn + 4) * g * (np.abs(F).T @ top)
    eF = ez @ np.abs(X).T + 1.001 * (t + 4) * g * (top @ np.abs(X).T)
    eb = es.sum(1) + 1.001 * (t + 4) * g * (np.abs(dz) + es).sum(1)
    return tuple(e + u * (np.abs(r) + e) + TINY[dtype] for e, r in ((eX, dX), (eF, dF), (eb, db)))

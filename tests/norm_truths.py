"""Plain 64-bit form of group norm with an activation, its gradients, and the error
bounds that follow from how the library computes them (torch only, no code of the
library).  Tensors are (c, s, b)."""
from __future__ import annotations

import math

import torch

UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}
ACT = {torch.float32: 2.0 ** -20, torch.bfloat16: 2.0 ** -15, torch.float16: 2.0 ** -15}    # an activation's own error
EPS = 2.0 ** -24
CHAIN = 300      # additions that a value passes in a sum: 256 in a thread or 16 and 128 in LDS, then trees


def value(z, act):
    if act == "relu":
        return torch.where(z <= 0, 0.0, z)
    if act == "gelu":
        return z * torch.erfc(-z / math.sqrt(2)) / 2
    if act == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    if act == "silu":
        return z * torch.sigmoid(z)
    return z


def slope(z, act):
    if act == "relu":
        return (z > 0).double()
    if act == "gelu":
        return torch.erfc(-z / math.sqrt(2)) / 2 + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":
        a = math.sqrt(2 / math.pi)
        t = torch.tanh(a * (z + 0.044715 * z ** 3))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * a * (1 + 3 * 0.044715 * z * z)
    if act == "silu":
        s = torch.sigmoid(z)
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)


def spread(v, groups, c):
    """(groups, b) to (c, 1, b)."""
    return v.double().repeat_interleave(c // groups, 0)[:, None]


def avg(v, groups):
    c, s, b = v.shape
    return v.reshape(groups, c // groups * s, b).mean(1)


def norm(x, groups, weight, bias, eps, act):
    x = x.double()
    c = x.shape[0]
    mean = avg(x, groups)
    var = avg((x - spread(mean, groups, c)) ** 2, groups)
    rstd = (var + eps) ** -0.5
    xhat = (x - spread(mean, groups, c)) * spread(rstd, groups, c)
    z = xhat * column(weight, c, 1.0, x) + column(bias, c, 0.0, x)
    return value(z, act), mean, rstd, xhat, z


def column(v, c, other, like):
    return (torch.full((c,), other, dtype=torch.float64, device=like.device) if v is None else v.double())[:, None, None]


def backward(x, dO, groups, weight, bias, eps, act):
    c = x.shape[0]
    _, _, rstd, xhat, z = norm(x, groups, weight, bias, eps, act)
    dz = torch.where(z <= 0, 0.0, dO.double()) if act == "relu" else dO.double() * slope(z, act)
    d = dz * column(weight, c, 1.0, x)
    dI = spread(rstd, groups, c) * (d - spread(avg(d, groups), groups, c) - xhat * spread(avg(d * xhat, groups), groups, c))
    return dI, (dz * xhat).sum((1, 2)), dz.sum((1, 2))


def bounds(x, groups, weight, bias, eps, act, dO=None):
    """Bounds of (O, mean, rstd), and with dO of (dI, dweight, dbias) behind them.

    The mean: CHAIN additions of |x|.  The squares: around the mean, or around a value of
    a thread's own, joined by the means: CHAIN additions of at most twice the largest
    square, and the mean's error squared.  xhat and Z follow; the activation's slope is at
    most 1.13 and its curvature 1; relu's slope may fall on either side where |Z| is
    within its error."""
    dtype, c = x.dtype, x.shape[0]
    o, mean, rstd, xhat, z = norm(x, groups, weight, bias, eps, act)
    xd = x.double()
    n = c // groups * x.shape[1]
    u, tiny = UNIT[dtype], TINY[dtype]
    e_mean = (min(CHAIN, n + 2) + 4) * EPS * avg(xd.abs(), groups)
    far = (xd - spread(mean, groups, c)).abs().reshape(groups, -1, x.shape[2]).amax(1)
    var = rstd ** -2 - eps
    e_var = (min(CHAIN, n + 2) + 8) * EPS * (var + torch.minimum(far ** 2, n * var)) + 4 * e_mean * EPS * far + 2 * e_mean ** 2 + tiny
    rel = 0.5 * e_var * rstd ** 2 + (e_var * rstd ** 2) ** 2 + 4 * EPS          # of rstd
    e_xhat = spread(rstd, groups, c) * (spread(e_mean, groups, c) + 2 * EPS * (xd - spread(mean, groups, c)).abs()) + xhat.abs() * spread(rel, groups, c)
    w, b = column(weight, c, 1.0, x).abs(), column(bias, c, 0.0, x).abs()
    e_z = w * e_xhat + 4 * EPS * (w * xhat.abs() + b)
    e_o = 1.13 * e_z + (0 if act == "none" else ACT[dtype] * z.abs())
    out = (e_o + u * (o.abs() + e_o) + tiny, e_mean + EPS * mean.abs(), rstd * rel + EPS * rstd)
    if dO is None:
        return out
    g = dO.double().abs()
    dI, dw, db = backward(x, dO, groups, weight, bias, eps, act)
    if act == "none":
        e_dz = torch.zeros_like(g)
        dz = dO.double()
    elif act == "relu":
        e_dz = torch.where(z.abs() <= e_z, g, 0.0)
        dz = torch.where(z <= 0, 0.0, dO.double())
    else:
        e_dz = g * (e_z + ACT[dtype] * (1 + z.abs()) + 2 * EPS)
        dz = dO.double() * slope(z, act)
    d, e_d = (dz * w).abs(), e_dz * w + 2 * EPS * dz.abs() * w
    dx, e_dx = d * xhat.abs(), e_d * xhat.abs() + d * e_xhat
    chain = (min(CHAIN, n + 2) + 8) * EPS
    ea, eax = avg(e_d, groups) + chain * avg(d + e_d, groups), avg(e_dx, groups) + chain * avg(dx + e_dx, groups)
    a, ax = avg(dz * column(weight, c, 1.0, x), groups).abs(), avg(dz * column(weight, c, 1.0, x) * xhat, groups).abs()
    up = lambda v: spread(v, groups, c)                                                # noqa: E731
    e_dI = up(rstd) * (e_d + up(ea) + xhat.abs() * up(eax) + e_xhat * up(ax + eax) + 8 * EPS * (d + up(a) + xhat.abs() * up(ax))) + dI.abs() * up(rel)
    long = (CHAIN + x.shape[2] + 8) * EPS
    e_dw = (e_dz * xhat.abs() + dz.abs() * e_xhat).sum((1, 2)) + long * (dz * xhat).abs().sum((1, 2))
    e_db = e_dz.sum((1, 2)) + long * dz.abs().sum((1, 2))
    return out + tuple(e + u * (r.abs() + e) + tiny for e, r in ((e_dI, dI), (e_dw, dw), (e_db, db)))

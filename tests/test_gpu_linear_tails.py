"""Activations and their slopes where they fall to nothing: within a few roundings
of themselves, not of z, down to the smallest normal values.  1 x 1 layers, whose
product is exact."""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

import layer_truths as lt64
from test_gpu_linear import DTYPES, host, lt, near, place

pytestmark = pytest.mark.gpu

ACTS = ["gelu", "gelu_tanh", "silu"]
K = math.sqrt(2 / math.pi)
TINY = {"float32": 2.0 ** -149, "bfloat16": 2.0 ** -133, "float16": 2.0 ** -25}


def grid(dtype):
    z = np.concatenate([np.linspace(-14, 14, 5601), -np.geomspace(1e-5, 14, 600), np.geomspace(1e-5, 14, 600)])
    return host(torch.from_numpy(z).to(DTYPES[dtype]))


def gate_error(z, act, dtype):
    """(gate, its relative error): act(z) = z gate(z).  e = 2^-24, twice that where
    the hardware's exp and reciprocal are used.  An exponent w is off by a few e |w|
    (its own roundings), its exp by that and a few e more.
      gelu       Phi: fp32 erfc(-z / sqrt 2), its argument off by 2 e relative, which
                 erfc magnifies by z^2 at most, its own 4 e and the products'; 16-bit:
                 2.8e-5 of the fit below z = 0, and above it of 1 - Phi <= Phi
      gelu_tanh  (1 + tanh u) / 2 = 1 / (1 + exp(-2u)), here too, since 1 + tanh u has
                 lost its digits below z = -5 even in 64 bits: the exponent off by 6 e |2u|
      silu       1 / (1 + exp(-z)): the exponent off by 3 e |z|"""
    e = 2.0 ** -24 if dtype == "float32" else 2.0 ** -23
    if act == "gelu":
        return lt64.phi(z), (8 + 3 * z * z) * e + (0 if dtype == "float32" else 2.8e-5)
    w = 2 * K * (z + 0.044715 * z ** 3) if act == "gelu_tanh" else z
    g = 1 / (1 + np.exp(-w))
    return g, ((6 if act == "gelu_tanh" else 3) * np.abs(w) + 4) * e * (1 - g) + 4 * e


def floor(factor):
    """exp(-w) leaves the range at w = -88.7 and the gate is taken for 0 there: what
    is lost of `factor` times a gate of exp(-88.7) < 2^-127, or, by the hardware's
    reciprocal of what is above 2^126, below 2^-126."""
    return factor * 2.0 ** -126


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("act", ACTS)
def test_values(act, dtype):
    z = grid(dtype)
    one = place(np.ones((1, 1)), DTYPES[dtype])
    gate, rel = gate_error(z, act, dtype)
    want = z * gate
    err = np.abs(z) * gate * (rel + 2 * 2.0 ** -24) + floor(np.abs(z))
    u = lt64.UNIT[dtype]
    near(lt().linear(one, place(z[None, :], DTYPES[dtype]), activation=act), want[None, :],
         (err + u * (np.abs(want) + err) + TINY[dtype])[None, :], act)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("act", ACTS)
def test_slopes(act, dtype):
    """dX of a 1 x 1 layer with dO = 4096, so that fp16 shows slopes of 1e-8: the
    slope's terms with their gates' errors, two roundings (dZ and dX)."""
    z = grid(dtype)
    d = 4096.0
    gate, rel = gate_error(z, act, dtype)
    e = 2.0 ** -24 if dtype == "float32" else 2.0 ** -23
    if act == "gelu":                              # Phi + z phi
        second = z * np.exp(-z * z / 2) / math.sqrt(2 * math.pi)
        err = gate * rel + np.abs(second) * (8 + 2 * z * z) * e
        lost = floor(1 + np.abs(z))
    else:                                          # g + w' z g (1 - g), w' the exponent's derivative
        slope = 2 * K * (1 + 3 * 0.044715 * z * z) if act == "gelu_tanh" else 1.0
        second = slope * z * gate * (1 - gate)
        err = gate * rel + np.abs(second) * (rel + 8 * e) + slope * np.abs(z) * gate * (gate * rel + e)
        lost = floor(1 + slope * np.abs(z))
    err = d * (err + 4 * e * np.abs(gate + second) + lost)
    want = d * (gate + second)
    u = lt64.UNIT[dtype]
    dz = err + u * (np.abs(want) + err) + TINY[dtype]
    one = place(np.ones((1, 1)), DTYPES[dtype])
    Z = place(z[None, :], DTYPES[dtype])
    dO = place(np.full((1, z.size), d), DTYPES[dtype])
    near(lt().linear_backward(one, Z, dO, pre=Z, activation=act, needs=(True, False, False))[0], want[None, :],
         (dz + u * (np.abs(want) + dz) + TINY[dtype])[None, :], act)

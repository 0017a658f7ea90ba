"""Argument checks of group norm's C ABI (``include/group_norm.h``), which come before any
GPU work (no GPU needed), and the plain form the GPU tests rest on."""
from __future__ import annotations

import os

import pytest
import torch

import norm_truths as truth
import paper_2005_06410_amd as lt
from paper_2005_06410_amd import build as ltbuild

BF16, F16, F32 = 4, 5, 1


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(lt.LIB_PATH):
        ltbuild.build()
    return lt.load()


SIZES = dict(dtype=F32, c=8, s=6, b=2, groups=4)
FORWARD = dict(SIZES, I=16, ldi=8, ldbi=48, weight=None, bias=None, eps=1e-5, act=0, O=16, ldo=8, ldbo=48, mean=None, rstd=None, ws=None,
               bytes=0, stream=None)
BACK = dict(SIZES, I=16, ldi=8, ldbi=48, dO=16, lddo=8, ldbdo=48, weight=None, bias=None, act=0, mean=16, rstd=16, dI=16, lddi=8, ldbdi=48,
            dweight=None, dbias=None, ws=16, bytes=1 << 40, stream=None)
SIZE_FAULTS = [({"dtype": 2}, -1), ({"c": -1}, -2), ({"c": 1 << 24}, -2), ({"s": -1}, -3), ({"s": 1 << 24}, -3), ({"b": -1}, -4), ({"b": 1 << 31}, -4),
               ({"c": 1 << 20, "s": 1 << 20}, -4), ({"groups": 0}, -5), ({"groups": 3}, -5), ({"groups": 16}, -5)]


@pytest.mark.parametrize("change,code", SIZE_FAULTS + [
    ({"I": None}, -6), ({"ldi": 7}, -7), ({"ldi": 1 << 40}, -7), ({"ldbi": 47}, -8), ({"eps": -1.0}, -11), ({"eps": float("nan")}, -11),
    ({"eps": 1e300}, -11), ({"act": 5}, -12), ({"act": -1}, -12), ({"O": None}, -13), ({"ldo": 7}, -14), ({"ldbo": 40}, -15),
    # chunks need their workspace
    ({"s": 1 << 20, "ldbi": 1 << 23, "ldbo": 1 << 23}, -18), ({"s": 1 << 20, "ldbi": 1 << 23, "ldbo": 1 << 23, "ws": 8}, -18),
    ({"s": 1 << 20, "ldbi": 1 << 23, "ldbo": 1 << 23, "ws": 16}, -19),
    ({"b": 0, "I": None, "O": None}, 0), ({"s": 0, "I": None, "O": None}, 0),
])
def test_argument_checks(lib, change, code):
    assert lib.convgemm_group_norm(*dict(FORWARD, **change).values()) == code


@pytest.mark.parametrize("change,code", SIZE_FAULTS + [
    ({"I": None}, -6), ({"ldi": 7}, -7), ({"ldbi": 47}, -8), ({"dO": None}, -9), ({"lddo": 7}, -10), ({"ldbdo": 47}, -11), ({"act": 5}, -14),
    ({"mean": None}, -15), ({"rstd": None}, -16), ({"lddi": 7}, -18), ({"ldbdi": 47}, -19), ({"ws": None}, -22), ({"ws": 8}, -22), ({"bytes": 8}, -23),
    ({"dI": None}, 0),
])
def test_backward_argument_checks(lib, change, code):
    assert lib.convgemm_group_norm_backward(*dict(BACK, **change).values()) == code


def test_workspace_queries(lib):
    for fn in (lib.convgemm_group_norm_workspace, lib.convgemm_group_norm_backward_workspace):
        assert fn(9, 8, 6, 2, 4) == -1 and fn(F32, 8, 6, 2, 3) == -5 and fn(F32, 8, 0, 2, 4) == 0
    assert lib.convgemm_group_norm_workspace(F32, 384, 169, 1, 32) == 0
    # far less than the maps
    assert lib.convgemm_group_norm_backward_workspace(BF16, 128, 65536, 16, 32) < 8 << 20


def test_the_plain_form_is_torchs():
    """Against torch's own group norm and automatic differentiation in 64 bits."""
    g = torch.Generator().manual_seed(1)
    for c, s, b, groups in [(12, 7, 3, 4), (5, 4, 2, 1), (6, 3, 2, 6)]:
        for act, fn in [("none", lambda v: v), ("relu", torch.relu), ("gelu", torch.nn.functional.gelu), ("silu", torch.nn.functional.silu),
                        ("gelu_tanh", lambda v: torch.nn.functional.gelu(v, approximate="tanh"))]:
            x, w, bias = (torch.randn(n, generator=g, dtype=torch.float64).requires_grad_() for n in ((b, c, s), (c,), (c,)))
            d = torch.randn(b, c, s, generator=g, dtype=torch.float64)
            want = fn(torch.nn.functional.group_norm(x, groups, w, bias, 1e-5))
            grads = torch.autograd.grad((want * d).sum(), [x, w, bias])
            x3, d3 = x.detach().permute(1, 2, 0), d.permute(1, 2, 0)
            got = truth.norm(x3, groups, w.detach(), bias.detach(), 1e-5, act)[0]
            assert (got - want.detach().permute(1, 2, 0)).abs().max() < 1e-12
            for a, v in zip(truth.backward(x3, d3, groups, w.detach(), bias.detach(), 1e-5, act), (grads[0].permute(1, 2, 0), *grads[1:])):
                assert (a - v).abs().max() < 1e-10

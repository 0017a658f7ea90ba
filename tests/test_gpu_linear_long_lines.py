"""Layers with millions of outputs or inputs: lines as long as that on both sides
of what the direct loads reach.  Sums of small integers, exact in every type."""
from __future__ import annotations

import pytest
import torch

from test_gpu_linear_kernels import ints, lt, same

pytestmark = pytest.mark.gpu


def sparse(gen, shape, per_line, dtype, order=0):
    """ints() with about `per_line` nonzero values in each line."""
    return ints(gen, shape, min(1.0, per_line / shape[0 if order == 0 else 1]), dtype, order=order)


@pytest.mark.parametrize("dtype,kn,ci,t", [
    (torch.bfloat16, 1 << 22, 64, 80), (torch.bfloat16, 1 << 22, 64, 8), (torch.float16, 5000001, 24, 128),
    (torch.float32, 2200000, 24, 128), (torch.float32, (1 << 21) - 2, 24, 40)])
@pytest.mark.parametrize("order", [0, 1])
@pytest.mark.parametrize("act", ["none", "relu"])
def test_many_outputs(dtype, kn, ci, t, order, act):
    """The library's own dZ has lines of kn values."""
    print(f"[many outputs] {dtype} {kn} x {ci}, {t} order {order} {act}", flush=True)
    g = torch.Generator(device="cuda")
    g.manual_seed(kn)
    F = ints(g, (kn, ci), 1.0, dtype, order=order)
    X = ints(g, (ci, t), 1.0, dtype)
    dO = sparse(g, (kn, t), 40, dtype)
    Z = ints(g, (kn, t), 1.0, dtype)
    dX, dF, db = lt().linear_backward(F, X, dO, pre=Z, activation=act)
    d = dO.double() * (Z > 0) if act == "relu" else dO.double()
    same(dX, F.double().t() @ d, "dX")
    same(dF, d @ X.double().t(), "dF")
    same(db, d.sum(1), "dbias")

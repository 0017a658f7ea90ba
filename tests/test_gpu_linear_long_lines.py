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


@pytest.mark.parametrize("dtype,kn,ci,t", [
    # on both sides of what the direct loads reach, with large and small tiles, few tokens and many
    (torch.bfloat16, 136, (1 << 23) - 8, 72), (torch.bfloat16, 136, (1 << 23) + 8, 72), (torch.float16, 130, 10000001, 70),
    (torch.bfloat16, 300, 9000000, 5), (torch.float32, 200, (1 << 22) - 4, 130), (torch.float32, 200, (1 << 22) + 4, 130),
    (torch.float32, 64, 5000003, 17), (torch.bfloat16, 9000000, 24, 100), (torch.float16, (1 << 24) - 1, 9, 66),
    (torch.float32, 4500001, 40, 129)])
@pytest.mark.parametrize("order", [0, 1])
def test_long_extents(dtype, kn, ci, t, order):
    print(f"[long extents] {dtype} {kn} x {ci}, {t} order {order}", flush=True)
    g = torch.Generator(device="cuda")
    g.manual_seed(ci)
    F = ints(g, (kn, ci), min(1.0, 40 / ci, 40 / kn), dtype, order=order)
    X, dO = ints(g, (ci, t), 1.0, dtype), sparse(g, (kn, t), 40, dtype)
    f, x, d = F.double(), X.double(), dO.double()
    want = f @ x
    assert want.abs().max() < 256 and 0 < want.abs().sum()
    same(lt().linear(F, X), want, "O")
    del want
    dX, dF, db = lt().linear_backward(F, X, dO)
    same(dX, f.t() @ d, "dX")
    same(dF, d @ x.t(), "dF")
    same(db, d.sum(1), "dbias")


@pytest.mark.parametrize("dtype,ld", [(torch.bfloat16, (1 << 23) - 8), (torch.bfloat16, (1 << 23) + 8), (torch.float32, (1 << 22) - 4)])
@pytest.mark.parametrize("order", [0, 1])
@pytest.mark.parametrize("t", [5, 700])
def test_lines_at_the_reach(dtype, ld, order, t):
    """Short lines, as far apart as the direct loads reach, and farther."""
    g = torch.Generator(device="cuda")
    g.manual_seed(ld)
    F = torch.full((ld * 300,), float("nan"), dtype=dtype, device="cuda").as_strided((300, 96), (ld, 1))
    F.copy_(ints(g, (300, 96), 0.2, torch.float32))
    F = F if order else F.t()
    X, dO = ints(g, (F.shape[1], t), 1.0, dtype), ints(g, (F.shape[0], t), 0.02, dtype)
    same(lt().linear(F, X), F.double() @ X.double(), "O")
    dX, dF, _ = lt().linear_backward(F, X, dO)
    same(dX, F.double().t() @ dO.double(), "dX")
    same(dF, dO.double() @ X.double().t(), "dF")

"""The layer's gradients one by one: what is left out changes neither what the call
needs nor what the others are."""
from __future__ import annotations

import itertools

import pytest
import torch

from test_gpu_linear_kernels import ints, lt, same

pytestmark = pytest.mark.gpu

SIZES = [(2070, 246, 52), (5361, 186, 7), (1001, 515, 77), (300, 9, 2000), (16, 2048, 40)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("order", [0, 1])
@pytest.mark.parametrize("act", ["none", "relu"])
@pytest.mark.parametrize("kn,ci,t", SIZES)
def test_every_subset(kn, ci, t, act, order, dtype):
    """Leading dimensions of whole vectors, extents of any length."""
    g = torch.Generator(device="cuda")
    g.manual_seed(kn)

    def some(shape, density, o=0):
        return ints(g, shape, density, dtype, pad=-shape[o] % 8, order=o)

    F, X = some((kn, ci), min(1.0, 40 / kn), order), some((ci, t), 1.0)
    dO, Z = some((kn, t), 40 / max(kn, t)), some((kn, t), 1.0)
    d = dO.double() * (Z > 0) if act == "relu" else dO.double()
    want = (F.double().t() @ d, d @ X.double().t(), d.sum(1))
    for needs in itertools.product((False, True), repeat=3):
        got = lt().linear_backward(F, X, dO, pre=Z, activation=act, needs=needs)
        for v, w, need in zip(got, want, needs):
            assert (v is not None) == need
            if need:
                same(v, w, f"{needs}")

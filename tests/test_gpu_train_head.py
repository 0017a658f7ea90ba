"""The example that runs the layer operators together: it learns, the same in
every type, and its gradients are those of torch's automatic differentiation."""
from __future__ import annotations

import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "train_head.py")


def example():
    spec = importlib.util.spec_from_file_location("train_head", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_the_head_learns(dtype):
    losses, norms = example().train(steps=40, dtype=dtype)
    assert all(n > 0 for n in norms)
    assert 1.5 < losses[0] < 4.5                      # about log 10 for scores near zero
    assert sum(losses[-5:]) / 5 < 0.3 * losses[0]


def test_gradients_are_autograds():
    """Two layers with residual against torch.autograd in 64 bits on the CPU: each
    fp32 result within K eps of sums of magnitude O(1) .. O(10)."""
    import paper_2005_06410_amd as lt
    g = torch.Generator().manual_seed(5)
    ci, h, t = 40, 24, 12
    F1, b1, F2 = (torch.randn(s, generator=g, dtype=torch.float64) for s in ((h, ci), (h,), (h, h)))
    x, w = torch.randn(t, ci, generator=g, dtype=torch.float64).t(), torch.randn(h, t, generator=g, dtype=torch.float64)
    dev = [v.float().cuda() for v in (F1, b1, F2)]
    X, W = (v.t().contiguous().float().cuda().t() for v in (x, w))
    leaves = [v.float().double().requires_grad_() for v in (F1, b1, F2, x)]
    a1 = torch.nn.functional.gelu(leaves[0] @ leaves[3] + leaves[1][:, None])
    out = torch.nn.functional.silu(leaves[2] @ a1) + a1
    (out * w.float().double()).sum().backward()
    h1, z1 = lt.linear(dev[0], X, bias=dev[1], activation="gelu", keep_pre=True)
    h2, z2 = lt.linear(dev[2], h1, activation="silu", residual=h1, keep_pre=True)
    dh1, dF2, _ = lt.linear_backward(dev[2], h1, W, pre=z2, activation="silu")
    dX, dF1, db1 = lt.linear_backward(dev[0], X, dh1 + W, pre=z1, activation="gelu")
    for got, want in ((h2, out), (dF1, leaves[0].grad), (db1, leaves[1].grad), (dF2, leaves[2].grad), (dX, leaves[3].grad)):
        want = want.detach()
        assert (got.double().cpu() - want).abs().max() <= 200 * 2.0 ** -24 * (1 + want.abs().max())

"""Trains the fully connected head of a small convolutional network with the
library's operators together: one CONVGEMM layer and its ``group_norm`` make the
features, two ``linear`` layers (GELU, SiLU and a residual) come before the classes,
whose scores ``linear_cross_entropy`` never writes; its gradients and
``linear_backward`` lead back, and ``clip_grad_norm`` bounds the step.  Images and
labels are synthetic: each class has a pattern of its own, and the images are noisy
copies.

    python examples/train_head.py [--steps 60] [--dtype bf16|f16|f32]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2005_06410_amd as lt  # noqa: E402

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def leftmost_fastest(shape, gen, scale):
    """Normal values stored with the leftmost index fastest."""
    t = torch.randn(tuple(reversed(shape)), generator=gen, device="cuda") * scale
    return t.permute(*reversed(range(len(shape))))


def features(images, filters):
    """(ci, batch) features: one convolution with stride 2, normalised in groups of
    four channels, relu, flattened."""
    o = lt.convgemm(filters, images, stride=2)            # (kn, ho, wo, batch), leftmost fastest
    kn, ho, wo, b = o.shape
    o, _, _ = lt.group_norm(o, kn // 4, activation="relu", out=o)
    return o.as_strided((kn * ho * wo, b), (1, kn * ho * wo))


def train(steps=60, dtype="bf16", classes=10, batch=64, hidden=256, rate=0.5, max_norm=1.0, seed=0):
    """The losses of the steps (host floats, read once at the end) and the norms
    of their gradients."""
    d = DTYPES[dtype]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    patterns = leftmost_fastest((15, 15, 3, classes), gen, 1.0)
    filters = leftmost_fastest((16, 3, 3, 3), gen, (2.0 / 27) ** 0.5)
    ci = 16 * 7 * 7
    # master copies in fp32; F is (outputs, inputs) with the inputs fastest
    master = [torch.randn(hidden, ci, generator=gen, device="cuda") * ci ** -0.5, torch.zeros(hidden, device="cuda"),
              torch.randn(hidden, hidden, generator=gen, device="cuda") * hidden ** -0.5, torch.zeros(hidden, device="cuda"),
              torch.randn(classes, hidden, generator=gen, device="cuda") * hidden ** -0.5, torch.zeros(classes, device="cuda")]
    mean = torch.full((), 1.0 / batch, device="cuda")                    # dL/dloss of every image
    losses, norms = [], []
    for _ in range(steps):
        label = torch.randint(0, classes, (batch,), generator=gen, device="cuda")
        images = patterns.permute(3, 2, 1, 0)[label] + 0.5 * torch.randn(batch, 3, 15, 15, generator=gen, device="cuda")
        x = features(images.contiguous().permute(3, 2, 1, 0), filters).to(d)
        F1, b1, F2, b2, F3, b3 = (p.to(d) for p in master)
        h1, z1 = lt.linear(F1, x, bias=b1, activation="gelu", keep_pre=True)
        h2, z2 = lt.linear(F2, h1, bias=b2, activation="silu", residual=h1, keep_pre=True)
        loss, lse = lt.linear_cross_entropy(F3, h2, label, bias=b3)
        losses.append(loss.mean())
        dh2, dF3, db3 = lt.linear_cross_entropy_backward(F3, h2, label, lse, mean, bias=b3)
        dh1, dF2, db2 = lt.linear_backward(F2, h1, dh2, pre=z2, activation="silu")
        _, dF1, db1 = lt.linear_backward(F1, x, dh1 + dh2, pre=z1, activation="gelu", needs=(False, True, True))
        grads = [dF1, db1, dF2, db2, dF3, db3]
        norms.append(lt.clip_grad_norm(grads, max_norm))
        for m, g in zip(master, grads):
            m.sub_(g.float(), alpha=rate)
    return [float(v) for v in torch.stack(losses)], [float(v) for v in torch.stack(norms)]


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--dtype", choices=sorted(DTYPES), default="bf16")
    a = ap.parse_args()
    losses, norms = train(a.steps, a.dtype)
    for i in range(0, a.steps, max(1, a.steps // 10)):
        print(f"step {i:4d}  loss {losses[i]:.4f}  gradient norm {norms[i]:.4f}")
    print(f"last       loss {losses[-1]:.4f}  gradient norm {norms[-1]:.4f}")


if __name__ == "__main__":
    main()

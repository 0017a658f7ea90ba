"""Results that would be written over what is still read are refused; neighbours in
one buffer and the overlaps that the operators allow are not."""
from __future__ import annotations

import pytest
import torch

from test_gpu_linear_kernels import ints, lt, same

pytestmark = pytest.mark.gpu


def gen():
    return torch.Generator(device="cuda").manual_seed(2)


def columns(flat, at, rows, cols, ld):
    return flat.as_strided((rows, cols), (1, ld), at)


def test_out_over_an_input_is_refused():
    g = gen()
    flat = torch.zeros(4096, device="cuda")
    X, F = columns(flat, 0, 16, 20, 16), ints(g, (16, 16), 1.0, torch.float32)
    R = columns(flat, 1024, 16, 20, 16)
    bias = flat[2048:2064]
    bad = [dict(out=X), dict(out=columns(flat, 16 * 19, 16, 20, 16)), dict(out=columns(flat, 8, 16, 20, 24)),
           dict(residual=R, out=columns(flat, 1024 + 16, 16, 20, 16)), dict(residual=R, out=columns(flat, 1024, 16, 20, 20)),
           dict(bias=bias, out=columns(flat, 2040, 16, 20, 16))]
    for kw in bad:
        with pytest.raises(ValueError):
            lt().linear(F, X, **kw)
    W = columns(flat, 0, 16, 16, 16)
    for f in (W, W.t()):
        with pytest.raises(ValueError):
            lt().linear(f, ints(g, (16, 20), 1.0, torch.float32), out=columns(flat, 255, 16, 20, 16))


def test_neighbours_and_the_residual_itself_are_taken():
    """The input's and the result's rows side by side in the same columns."""
    g = gen()
    flat = torch.zeros(4096, device="cuda")
    X, out, F = columns(flat, 0, 16, 20, 40), columns(flat, 16, 24, 20, 40), ints(g, (24, 16), 1.0, torch.float32)
    X.copy_(ints(g, (16, 20), 1.0, torch.float32))
    want = F.double() @ X.double()
    same(lt().linear(F, X, out=out), want, "neighbours")
    same(lt().linear(F, X, residual=out, out=out), 2 * want, "residual")
    same(lt().linear(F, X, out=columns(flat, 20 * 40, 24, 20, 24)), want, "behind")
    empty = columns(flat, 0, 16, 0, 16)
    assert lt().linear(ints(g, (16, 16), 1.0, torch.float32), empty, out=empty).shape == (16, 0)


def test_clipping_into_another_gradient_is_refused():
    a, b, e = torch.ones(8, device="cuda"), torch.ones(8, device="cuda"), torch.zeros(0, device="cuda")
    with pytest.raises(ValueError):
        lt().clip_grad_norm([a, b], 1.0, out=[b, a])
    with pytest.raises(ValueError):
        lt().clip_grad_norm([a, e, b], 1.0, out=[torch.empty_like(a), e, a])
    assert float(lt().clip_grad_norm([a, e, b], 2.0, out=[a, e, torch.empty_like(b)])) == 4.0
    assert (a == 0.5).all() and (b == 1.0).all()

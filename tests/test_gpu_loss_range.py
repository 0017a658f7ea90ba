"""The losses' gradients for incoming gradients of any size, and for infinite ones."""
from __future__ import annotations

import pytest
import torch

import loss_truths as truth
from test_gpu_loss import DTYPES, IGNORE, backward, forward, gen, labels_of, layer, teacher_of, within

pytestmark = pytest.mark.gpu


def cases(g, kn, t, dtype):
    yield {"labels": labels_of(g, kn, t), "ignore": IGNORE}
    top, index = teacher_of(g, kn, t, 5, dtype)
    yield {"top": top, "index": index, "temperature": 2.0}


@pytest.mark.parametrize("dtype,powers", [(torch.float32, (-60, 30, 100)), (torch.bfloat16, (-100, -60, 30, 100)), (torch.float16, (-9, 5))])
def test_gradients_follow_their_scale(dtype, powers):
    """2^k times the incoming gradient gives 2^k times the gradients, bit for bit: fp32 has room
    for what lies between, 16-bit types take the size out first (the factor that puts the largest at
    2^15 is then 2^-k times as large).  Left out is what the results' type rounds for its
    range."""
    g = gen(1)
    for kn, ci, t in [(900, 48, 64), (1000, 64, 1), (9000, 40, 33)]:
        F, X, b = layer(g, kn, ci, t, dtype, 1)
        for case in cases(g, kn, t, dtype):
            lse = forward(F, X, b, case)[1]
            gr = torch.rand(t, generator=g, device="cuda") + 0.5
            want = backward(F, X, b, case, lse, gr)
            for k in powers:
                got = backward(F, X, b, case, lse, gr * 2.0 ** k)
                for a, v in zip(got, want):
                    whole = v.double() * 2.0 ** k
                    # a zero may be a value that the type has no room for
                    tiny, most = torch.finfo(dtype).tiny, torch.finfo(dtype).max
                    inside = (v.abs() > tiny) & (whole.abs() > tiny) & (whole.abs() < most)
                    if dtype == torch.float32:        # its small dZ, 2^-60 of exponentials, may be rounded for their range
                        inside &= v.abs() > 2.0 ** -30
                    assert inside.any()
                    assert torch.equal(a.double()[inside], whole[inside]), f"2^{k}"


def test_gradients_below_the_factors_range():
    """16-bit types hold dZ times 2^15 over the largest |g| T, at most 2^15 / 1e-33: below, dZ is
    smaller, but bf16 has the range."""
    g = gen(2)
    F, X, b = layer(g, 900, 48, 64, torch.bfloat16, 0)
    for case in cases(g, 900, 64, torch.bfloat16):
        lse = forward(F, X, b, case)[1]
        base = torch.rand(64, generator=g, device="cuda") + 0.5
        for size in (1e-33, 1e-35, 1e-37):
            gr = base * size
            got = backward(F, X, b, case, lse, gr)
            for a, want, bound in zip(got, truth.backward(F, X, b, case, gr), truth.backward_bound(F, X, b, case, gr, torch.bfloat16)):
                within(a, want, bound, f"g about {size}")


@pytest.mark.parametrize("bad", [torch.inf, -torch.inf, torch.nan])
@pytest.mark.parametrize("dtype", DTYPES)
def test_an_infinite_gradient_stays_in_its_column(dtype, bad):
    """The factor is taken from the finite ones; the column's own dX, and what it adds to, is
    infinite or NaN, the other columns' dX are what they are without it."""
    g = gen(3)
    for kn, ci, t in [(900, 48, 64), (3000, 64, 9)]:
        F, X, b = layer(g, kn, ci, t, dtype, 1)
        for case in cases(g, kn, t, dtype):
            if "labels" in case:
                case["labels"][1] = 7
            lse = forward(F, X, b, case)[1]
            gr = torch.rand(t, generator=g, device="cuda") + 0.5
            without, beside = gr.clone(), gr.clone()
            without[1], beside[1] = 0.0, bad
            want, got = backward(F, X, b, case, lse, without), backward(F, X, b, case, lse, beside)
            keep = torch.arange(t, device="cuda") != 1
            assert torch.equal(got[0][:, keep], want[0][:, keep]) and not want[0][:, 1].any()
            assert not got[0][:, 1].isfinite().any() and not got[1].isfinite().any() and not got[2].isfinite().any()

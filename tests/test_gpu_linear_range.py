"""The layer's fp16 gradients where dZ leaves the range of fp16 and the gradients do
not: dO near the largest value under a slope above one, dO among the smallest
values under a slope below one, and values that are not finite beside them."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import layer_truths as lt64
from test_gpu_linear import host, lt, near, place, rng

pytestmark = pytest.mark.gpu

U, ACT, F16 = 2.0 ** -11, lt64.ACT["float16"], torch.float16


def bounds(F, X, dO, z, act):
    """Bounds of dX, dF and dbias.  dZ carries the slope's error (ACT (1 + |z|)
    |dO|), one rounding of fp16 and, held times a power of two that puts the
    largest |dO| at 2^14 at least, an absolute error of 2^-25 / 2^14 of that |dO|;
    then fp32 sums and one rounding of each result (half of fp16's spacing near
    zero, 2^-24, where it is below the normal range)."""
    dX, dF, db, dz = lt64.backward(F, X, dO, z, act)
    es = (ACT * (1 + np.abs(z)) + 2.0 ** -24) * np.abs(dO)
    ez = es + U * (np.abs(dz) + es) + 2.0 ** -39 * np.abs(dO).max()
    top = np.abs(dz) + ez
    g = 1.001 * 2.0 ** -24
    eX = np.abs(F).T @ ez + (F.shape[0] + 4) * g * (np.abs(F).T @ top)
    eF = ez @ np.abs(X).T + (X.shape[1] + 4) * g * (top @ np.abs(X).T)
    eb = es.sum(1) + (X.shape[1] + 4) * g * (np.abs(dz) + es).sum(1)
    return tuple(e + U * (np.abs(r) + e) + 2.0 ** -25 for e, r in ((eX, dX), (eF, dF), (eb, db)))


def check(F, X, dO, z, act, needs=(True, True, True)):
    got = lt().linear_backward(F, X, dO, pre=z, activation=act, needs=needs)
    h = [host(v) for v in (F, X, dO, z)]
    for g, w, b, name in zip(got, lt64.backward(*h, act), bounds(*h, act), ("dX", "dF", "dbias")):
        if g is not None:
            assert np.abs(w).max() < 60000
            near(g, w, b, name)


SMOOTH = ["gelu", "gelu_tanh", "silu"]


@pytest.mark.parametrize("act", SMOOTH)
@pytest.mark.parametrize("order", [0, 1])
@pytest.mark.parametrize("kn,ci,t", [(8, 8, 8), (203, 131, 70), (264, 72, 5), (520, 300, 300)])
def test_large_gradients(kn, ci, t, order, act):
    """dO up to fp16's largest value where the slope is above one."""
    r = rng(21, kn)
    F = place(r.standard_normal((kn, ci)) * 2.0 ** -9, F16, order=order)
    X = place(r.standard_normal((ci, t)) * 2.0 ** -9, F16)
    z = place(r.uniform(1.2, 2.6, (kn, t)), F16)
    dO = place(r.choice([-1.0, 1.0], (kn, t)) * r.uniform(40000, 65504, (kn, t)), F16)
    check(F, X, dO, z, act, needs=(True, True, False))          # dbias itself may leave the range


@pytest.mark.parametrize("act", SMOOTH)
@pytest.mark.parametrize("order", [0, 1])
@pytest.mark.parametrize("kn,ci,t", [(8, 8, 8), (203, 131, 70), (264, 72, 5), (520, 300, 300)])
@pytest.mark.parametrize("size", [2.0 ** -21, 2.0 ** -18, 2.0 ** -13])
def test_small_gradients(size, kn, ci, t, order, act):
    """dO of a few of fp16's smallest steps: dZ is not rounded to them."""
    r = rng(22, kn)
    F = place(r.standard_normal((kn, ci)) * 64, F16, order=order)
    X = place(r.standard_normal((ci, t)) * 64, F16)
    check(F, X, place(r.standard_normal((kn, t)) * size, F16), place(r.standard_normal((kn, t)), F16), act)


@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan])
def test_beside_values_that_are_not_finite(bad):
    """An infinite or NaN dO reaches its own token's dX and its own row's dF and
    dbias; it does not choose the factor of the others."""
    r = rng(23)
    kn, ci, t = 130, 70, 33
    F, X, z = (place(r.standard_normal(s) * 64, F16) for s in ((kn, ci), (ci, t), (kn, t)))
    d = r.standard_normal((kn, t)) * 2.0 ** -20
    clean = place(d, F16)
    d[17, 5] = bad
    dX, dF, db = (host(v) for v in lt().linear_backward(F, X, place(d, F16), pre=z, activation="silu"))
    h = [host(v) for v in (F, X, clean, z)]
    (wX, wF, wb, _), (eX, eF, eb) = lt64.backward(*h, "silu"), bounds(*h, "silu")
    tok, row = np.arange(t) != 5, np.arange(kn) != 17
    assert not np.isfinite(dX[:, 5]).any() and not np.isfinite(dF[17]).any() and not np.isfinite(db[17])
    for g, w, e in ((dX[:, tok], wX[:, tok], eX[:, tok]), (dF[row], wF[row], eF[row]), (db[row], wb[row], eb[row])):
        assert np.isfinite(g).all() and (np.abs(g - w) <= e).all()


def test_all_zero():
    F, X, z = (place(np.ones(s), F16) for s in ((40, 24), (24, 9), (40, 9)))
    for g in lt().linear_backward(F, X, place(np.zeros((40, 9)), F16), pre=z, activation="gelu"):
        assert not host(g).any()


def test_the_factor_follows_the_gradients():
    """Captured once and replayed with gradients of other sizes, eager work between
    the replays: the factor is that of the call's own dO, on any stream."""
    r = rng(24)
    kn, ci, t = 264, 136, 40
    F, X, z = (place(r.standard_normal(s), F16) for s in ((kn, ci), (ci, t), (kn, t)))
    d = r.standard_normal((kn, t))
    dO = place(d, F16)

    def call():
        return lt().linear_backward(F, X, dO, pre=z, activation="gelu")

    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = call()
    side = torch.cuda.Stream()
    for size in (2.0 ** -20, 8.0, 2.0 ** -8, 2.0 ** -20):
        dO.copy_(torch.from_numpy(d * size).to(F16))
        g.replay()
        torch.cuda.synchronize()
        replayed = [v.clone() for v in got]
        eager = call()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            other = call()
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        h = [host(v) for v in (F, X, dO, z)]
        for a, b, c, want, bound, name in zip(replayed, eager, other, lt64.backward(*h, "gelu"), bounds(*h, "gelu"), ("dX", "dF", "dbias")):
            assert torch.equal(a, b) and torch.equal(b, c), (size, name)
            near(a, want, bound, name)

"""The layer operators on the GPU against plain 64-bit forms: types, orders of
the weights, sizes from nothing to several tiles and ragged everywhere, leading
dimensions with NaN in the gaps, unaligned addresses, every activation."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import layer_truths as lt64

pytestmark = pytest.mark.gpu

DTYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}


def lt():
    import paper_2005_06410_amd as m
    return m


def rng(*seed):
    return np.random.default_rng(seed)


def place(a, dtype, ld=None, shift=0, order=0):
    """`a` (2-D, float64) on the GPU, first index fastest (order 0) or last
    (order 1), lines `ld` apart and `shift` values into its memory; every value
    around it is NaN.  Returns the view; its values are exactly `a` rounded."""
    m = a if order == 0 else a.T
    rows, cols = m.shape
    ld = max(rows, 1) if ld is None else ld
    flat = torch.full((shift + ld * max(cols, 1) + 8,), float("nan"), dtype=dtype, device="cuda")
    v = flat[shift:shift + ld * max(cols, 1)].as_strided((rows, cols), (1, ld), shift)
    if a.size:
        v.copy_(torch.from_numpy(np.ascontiguousarray(m)).to(dtype))
    return v if order == 0 else v.t()


def host(t):
    return t.detach().to(torch.float64).cpu().numpy()


def near(got, want, bound, what):
    got = host(got)
    assert got.shape == want.shape, what
    if not want.size:
        return
    assert np.isfinite(got).all(), f"{what}: not finite"
    worst = np.max(np.abs(got - want) / bound)
    assert worst <= 1.0, f"{what}: {worst:.3g} times the bound"


def layer(kn, ci, t, dtype, seed, order=0, pad=0, shift=0, bias=True, residual=True):
    r = rng(seed, kn, ci, t)
    d = DTYPES[dtype]

    def some(a, o=0):
        rows = a.shape[o]
        return place(a, d, max(rows, 1) + pad, shift, o)

    F = some(r.standard_normal((kn, ci)) / max(ci, 1) ** 0.5, order)
    X = some(r.standard_normal((ci, t)))
    b = some(0.5 * r.standard_normal((kn, 1)))[:, 0] if bias else None
    R = some(r.standard_normal((kn, t))) if residual else None
    return F, X, b, R


SIZES = [(1, 1, 1), (5, 3, 2), (16, 64, 1), (64, 64, 64), (130, 129, 3), (128, 256, 128), (257, 65, 131), (1001, 515, 77),
         (96, 1000, 300), (512, 2048, 16), (300, 1536, 33), (1024, 384, 520)]


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("order", [0, 1])
@pytest.mark.parametrize("kn,ci,t", SIZES)
def test_linear_sizes(kn, ci, t, order, dtype):
    print(f"[linear] {dtype} {kn} {ci} {t} order {order}", flush=True)
    F, X, b, R = layer(kn, ci, t, dtype, 1, order)
    h = [host(v) for v in (F, X, b, R)]
    O, Z = lt().linear(F, X, bias=b, activation="gelu", residual=R, keep_pre=True)
    want, z = lt64.linear(h[0], h[1], h[2], "gelu", h[3])
    bo, bz = lt64.linear_bound(h[0], h[1], h[2], "gelu", h[3], dtype)
    near(Z, z, bz, "Z")
    near(O, want, bo, "O")
    assert O.stride() == (1, kn) and torch.equal(O, lt().linear(F, X, bias=b, activation="gelu", residual=R))


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("act", lt64.ACTS)
@pytest.mark.parametrize("bias,residual", [(False, False), (True, False), (False, True)])
def test_linear_epilogues(act, bias, residual, dtype):
    F, X, b, R = layer(200, 96, 40, dtype, 2, 1, bias=bias, residual=residual)
    h = [None if v is None else host(v) for v in (F, X, b, R)]
    near(lt().linear(F, X, bias=b, activation=act, residual=R), lt64.linear(h[0], h[1], h[2], act, h[3])[0],
         lt64.linear_bound(h[0], h[1], h[2], act, h[3], dtype)[0], act)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("order", [0, 1])
@pytest.mark.parametrize("pad,shift", [(8, 0), (3, 0), (0, 1), (8, 8), (5, 3)])
@pytest.mark.parametrize("kn,ci,t", [(136, 200, 72), (131, 203, 70), (264, 72, 5), (1030, 130, 1)])
def test_linear_gaps_and_alignment(kn, ci, t, pad, shift, order, dtype):
    """NaN in every gap: a value read from one would show."""
    print(f"[linear gaps] {dtype} {kn} {ci} {t} order {order} pad {pad} shift {shift}", flush=True)
    F, X, b, R = layer(kn, ci, t, dtype, 3, order, pad, shift)
    h = [host(v) for v in (F, X, b, R)]
    out = place(np.zeros((kn, t)), DTYPES[dtype], kn + pad, shift)
    around = out.untyped_storage().nbytes()
    flat = torch.empty(0, dtype=DTYPES[dtype], device="cuda").set_(out.untyped_storage())
    before = torch.isnan(flat).sum()
    got = lt().linear(F, X, bias=b, activation="silu", residual=R, out=out)
    assert got is out and out.untyped_storage().nbytes() == around
    near(out, lt64.linear(h[0], h[1], h[2], "silu", h[3])[0], lt64.linear_bound(h[0], h[1], h[2], "silu", h[3], dtype)[0], "O")
    assert torch.isnan(flat).sum() == before, "a gap of the output was written"


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("order", [0, 1])
@pytest.mark.parametrize("kn,ci,t", [(64, 96, 8), (333, 250, 17), (1040, 130, 1), (150, 2050, 140), (700, 640, 513)])
def test_linear_exact_on_integers(kn, ci, t, order, dtype):
    """Sums of small integers are exact in any order of summation."""
    r = rng(4, kn, ci, t)
    d = DTYPES[dtype]
    F = place((r.random((kn, ci)) < 0.05) * r.integers(-1, 2, (kn, ci)).astype(float), d, order=order)
    X = place(r.integers(-1, 2, (ci, t)).astype(float), d)
    want = host(F) @ host(X)
    assert np.abs(want).max() <= 256
    assert np.array_equal(host(lt().linear(F, X)), want)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("order", [0, 1])
def test_linear_empty(order, dtype):
    d = DTYPES[dtype]
    r = rng(5)
    # no inputs: a product over no terms is zero, the epilogue still holds
    F, X = place(np.zeros((70, 0)), d, order=order), place(np.zeros((0, 9)), d)
    b, R = place(r.standard_normal((70, 1)), d)[:, 0], place(r.standard_normal((70, 9)), d)
    hb, hr = host(b), host(R)
    near(lt().linear(F, X, bias=b, activation="relu", residual=R), np.maximum(hb, 0)[:, None] + hr,
         lt64.linear_bound(np.zeros((70, 0)), np.zeros((0, 9)), hb, "relu", hr, dtype)[0], "no inputs")
    # no tokens, no outputs
    F, X = place(np.ones((70, 5)), d, order=order), place(np.zeros((5, 0)), d)
    assert lt().linear(F, X).shape == (70, 0)
    F, X = place(np.zeros((0, 5)), d, order=order), place(np.ones((5, 3)), d)
    assert lt().linear(F, X).shape == (0, 3)
    # their gradients
    F, X, dO = place(np.ones((70, 5)), d, order=order), place(np.zeros((5, 0)), d), place(np.zeros((70, 0)), d)
    dX, dF, db = lt().linear_backward(F, X, dO, pre=dO, activation="silu")
    assert dX.shape == (5, 0) and not host(dF).any() and not host(db).any() and dF.shape == (70, 5) and db.shape == (70,)
    F, X, dO = place(np.zeros((0, 5)), d, order=order), place(np.ones((5, 3)), d), place(np.zeros((0, 3)), d)
    dX, dF, db = lt().linear_backward(F, X, dO)
    assert dF.shape == (0, 5) and db.shape == (0,) and dX.shape == (5, 3) and not host(dX).any()


@pytest.mark.parametrize("act", lt64.ACTS)
def test_linear_infinities_and_nan(act):
    """One infinite and one NaN input reach their own columns only; the values
    follow the formula."""
    r = rng(6)
    F = place(np.abs(r.standard_normal((140, 64))) + 0.1, torch.float32)
    x = r.standard_normal((64, 6))
    x[5, 1], x[7, 2], x[9, 3] = np.inf, np.nan, -np.inf
    X = place(x, torch.float32)
    O = host(lt().linear(F, X, activation=act))
    with np.errstate(all="ignore"):
        want = lt64.linear(host(F), host(X), None, act, None)[0]
    assert np.array_equal(np.isnan(O), np.isnan(want)) and np.array_equal(np.isinf(O), np.isinf(want))
    assert np.isfinite(O[:, [0, 4, 5]]).all() and np.isnan(O[:, 2]).all() and (O[:, 1] == np.inf).all()


@pytest.mark.parametrize("act", lt64.ACTS)
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_activation_over_its_range(act, dtype):
    """A 1 x 1 layer is the activation itself: every magnitude, both signs."""
    z = np.concatenate([[0.0], np.geomspace(1e-6, 60, 400), np.linspace(0.01, 12, 700)])
    z = np.concatenate([z, -z])
    X = place(z[None, :], DTYPES[dtype])
    z = host(X)
    one = place(np.ones((1, 1)), DTYPES[dtype])
    near(lt().linear(one, X, activation=act), lt64.value(z, act),
         lt64.linear_bound(np.ones((1, 1)), z, None, act, None, dtype)[0], act)
    dO = place(np.ones_like(z), DTYPES[dtype])
    dX = lt().linear_backward(one, X, dO, pre=X, activation=act, needs=(True, False, False))[0]
    near(dX, lt64.backward(np.ones((1, 1)), z, np.ones_like(z), z, act)[0],
         lt64.backward_bound(np.ones((1, 1)), z, np.ones_like(z), z, act, dtype)[0], f"{act} slope")


BACKWARD_SIZES = [(1, 1, 1), (7, 5, 3), (64, 128, 16), (257, 131, 65), (300, 520, 77), (1001, 515, 130), (128, 64, 1030),
                  (1000, 1024, 80)]


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("order", [0, 1])
@pytest.mark.parametrize("act", ["none", "gelu"])
@pytest.mark.parametrize("kn,ci,t", BACKWARD_SIZES)
def test_backward_sizes(kn, ci, t, act, order, dtype):
    print(f"[backward] {dtype} {kn} {ci} {t} order {order} {act}", flush=True)
    F, X, _, dO = layer(kn, ci, t, dtype, 7, order)
    pre = layer(kn, ci, t, dtype, 8, order)[3]
    h = [host(v) for v in (F, X, dO, pre)]
    got = lt().linear_backward(F, X, dO, pre=pre, activation=act)
    want = lt64.backward(h[0], h[1], h[2], h[3], act)
    bound = lt64.backward_bound(h[0], h[1], h[2], h[3], act, dtype)
    for g, w, b, name in zip(got, want, bound, ("dX", "dF", "dbias")):
        near(g, w, b, name)
    assert got[1].stride() == F.stride() or min(kn, ci) == 1
    again = lt().linear_backward(F, X, dO, pre=pre, activation=act)
    assert all(torch.equal(a, b) for a, b in zip(got, again)), "not reproducible"


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("order", [0, 1])
@pytest.mark.parametrize("act", lt64.ACTS)
@pytest.mark.parametrize("pad,shift", [(8, 0), (3, 5)])
def test_backward_gaps_and_parts(act, order, pad, shift, dtype):
    kn, ci, t = 200, 136, 72
    F, X, _, dO = layer(kn, ci, t, dtype, 9, order, pad, shift)
    pre = layer(kn, ci, t, dtype, 10, order, pad, shift)[3]
    h = [host(v) for v in (F, X, dO, pre)]
    want = lt64.backward(h[0], h[1], h[2], h[3], act)
    bound = lt64.backward_bound(h[0], h[1], h[2], h[3], act, dtype)
    whole = lt().linear_backward(F, X, dO, pre=pre, activation=act)
    for needs in [(True, True, True), (True, False, False), (False, True, False), (False, False, True)]:
        got = lt().linear_backward(F, X, dO, pre=pre, activation=act, needs=needs)
        for g, w, b, full, need, name in zip(got, want, bound, whole, needs, ("dX", "dF", "dbias")):
            assert (g is None) == (not need)
            if need:
                near(g, w, b, name)
                assert torch.equal(g, full)


@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu"])
def test_gradient_against_differences(act):
    """dX, dF and dbias against central differences of sum(dO O) in 64 bits;
    the differences' own error is about h^2, the fp32 gradient's far less."""
    r = rng(11)
    kn, ci, t, h = 6, 5, 4, 1e-4
    F, X, b, dO = (place(r.standard_normal(s), torch.float32) for s in ((kn, ci), (ci, t), (kn, 1), (kn, t)))
    Fh, Xh, bh, dh = (host(v) for v in (F, X, b, dO))
    _, Z = lt().linear(F, X, bias=b[:, 0], activation=act, keep_pre=True)
    got = [host(v) for v in lt().linear_backward(F, X, dO, pre=Z, activation=act)]

    def loss(F_, X_, b_):
        return float((dh * lt64.linear(F_, X_, b_[:, 0], act, None)[0]).sum())

    for k, (base, g) in enumerate(zip((Xh, Fh, bh), (got[0], got[1], got[2][:, None]))):
        for at in np.ndindex(base.shape):
            up, down = base.copy(), base.copy()
            up[at] += h
            down[at] -= h
            args = [(Fh, up, bh), (up, Xh, bh), (Fh, Xh, up)][k], [(Fh, down, bh), (down, Xh, bh), (Fh, Xh, down)][k]
            want = (loss(*args[0]) - loss(*args[1])) / (2 * h)
            assert abs(g[at] - want) <= 1e-4 * (1 + abs(want))


def test_relu_gradient_where_dO_is_not_finite():
    """Masked values are zero whatever comes in."""
    z = place(np.array([[-1.0, 0.0, 2.0, 3.0]]), torch.float32)
    dO = place(np.array([[np.inf, np.nan, 5.0, -1.0]]), torch.float32)
    one = place(np.ones((1, 1)), torch.float32)
    dX, dF, db = lt().linear_backward(one, z, dO, pre=z, activation="relu")
    assert host(dX).tolist() == [[0.0, 0.0, 5.0, -1.0]] and host(db).tolist() == [4.0] and host(dF).tolist() == [[7.0]]


def test_residual_in_place():
    F, X, b, R = layer(96, 64, 33, "bfloat16", 12)
    want = lt().linear(F, X, bias=b, activation="silu", residual=R)
    assert lt().linear(F, X, bias=b, activation="silu", residual=R, out=R) is R and torch.equal(R, want)


def test_linear_is_the_convolution_of_one_position():
    """A 1 x 1 convolution on a 1 x 1 image, through the framework's other operator."""
    r = rng(13)
    F, X = place(r.standard_normal((64, 48)), torch.float32), place(r.standard_normal((48, 20)), torch.float32)
    O = lt().convgemm(F.as_strided((64, 1, 1, 48), (1, 64, 64, 64)), X.as_strided((1, 1, 48, 20), (1, 1, 1, 48)))
    near(lt().linear(F, X), host(O).reshape(64, 20), 2 * lt64.linear_bound(host(F), host(X), None, "none", None, "float32")[0], "conv")


def test_other_stream():
    """Work on a stream of its own, with its workspace."""
    F, X, b, R = layer(130, 4096, 70, "bfloat16", 14)
    want = lt().linear(F, X, bias=b, residual=R)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = [lt().linear(F, X, bias=b, residual=R) for _ in range(4)]
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    assert all(torch.equal(g, want) for g in got)


def test_graph_replays():
    """Captured once, replayed with new inputs, eager work between the replays."""
    F, X, b, R = layer(264, 2048, 24, "bfloat16", 15)
    dO = R.clone()
    lt().linear(F, X, bias=b, activation="gelu", residual=R, keep_pre=True)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        O, Z = lt().linear(F, X, bias=b, activation="gelu", residual=R, keep_pre=True)
        grads = lt().linear_backward(F, X, dO, pre=Z, activation="gelu")
        norm = lt().clip_grad_norm(grads, 1.0)
    for k in range(4):
        X.copy_(torch.randn(X.shape, device="cuda"))
        g.replay()
        torch.cuda.synchronize()
        got = [v.clone() for v in (O, Z, *grads, norm)]
        wO, wZ = lt().linear(F, X, bias=b, activation="gelu", residual=R, keep_pre=True)
        wg = lt().linear_backward(F, X, dO, pre=wZ, activation="gelu")
        wn = lt().clip_grad_norm(wg, 1.0)
        assert all(torch.equal(a, b_) for a, b_ in zip(got, (wO, wZ, *wg, wn))), k


def test_refusals():
    m = lt()
    f = torch.float32
    F, X = place(np.ones((6, 4)), f), place(np.ones((4, 3)), f)
    dO = place(np.ones((6, 3)), f)
    bad = [
        lambda: m.linear(F.cpu(), X.cpu()),
        lambda: m.linear(F.cpu(), X),
        lambda: m.linear(F, place(np.ones((5, 3)), f)),                    # ci differs
        lambda: m.linear(F, X.t().contiguous().t()[:, ::2][:, :1].expand(4, 3)),   # no stride along t
        lambda: m.linear(F, torch.ones(4, 3, device="cuda")),             # other order
        lambda: m.linear(F, X.double()),
        lambda: m.linear(F.half(), X),
        lambda: m.linear(F.double(), X.double()),
        lambda: m.linear(F[:, 0], X),
        lambda: m.linear(F, X[:, 0]),
        lambda: m.linear(F, X, bias=torch.ones(5, device="cuda")),
        lambda: m.linear(F, X, bias=torch.ones(12, device="cuda")[::2]),
        lambda: m.linear(F, X, bias=torch.ones(6, device="cuda").half()),
        lambda: m.linear(F, X, bias=torch.ones(6)),
        lambda: m.linear(F, X, activation="tanh"),
        lambda: m.linear(F, X, residual=torch.ones(3, 6, device="cuda")),
        lambda: m.linear(F, X, residual=dO.half()),
        lambda: m.linear(F, X, out=torch.ones(6, 3, device="cuda")),
        lambda: m.linear_backward(F, X, dO, activation="gelu"),           # no pre-activation
        lambda: m.linear_backward(F, X, torch.ones(6, 3, device="cuda")),
        lambda: m.linear_backward(F, X, dO, pre=dO.half(), activation="gelu"),
        lambda: m.linear_backward(F, X, dO[:, :2]),
        lambda: m.grad_norm([]),
        lambda: m.grad_norm([torch.ones(3)]),
        lambda: m.grad_norm([torch.ones(3, device="cuda"), torch.ones(3)]),
        lambda: m.grad_norm([torch.ones(3, device="cuda").double()]),
        lambda: m.grad_norm([torch.ones(6, device="cuda")[::2]]),
        lambda: m.grad_norm([torch.ones(1, device="cuda").expand(4)]),
        lambda: m.clip_grad_norm([dO], -1.0),
        lambda: m.clip_grad_norm([dO], float("nan")),
        lambda: m.clip_grad_norm([dO], 1.0, out=[dO, dO]),
        lambda: m.clip_grad_norm([dO], 1.0, out=[dO.half()]),
        lambda: m.clip_grad_norm([dO], 1.0, out=[torch.ones(6, 3, device="cuda")]),
    ]
    for i, call in enumerate(bad):
        with pytest.raises((ValueError, TypeError)):
            call()
            pytest.fail(f"refusal {i}")

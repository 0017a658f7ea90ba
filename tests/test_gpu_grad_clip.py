"""The joint norm of many gradients and clipping, on the GPU against 64-bit sums:
counts that need several launches, ragged and empty tensors, mixed types,
unaligned addresses, magnitudes whose squares leave the fp32 range."""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DTYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
UNIT = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}


def lt():
    import paper_2005_06410_amd as m
    return m


def host(t):
    return t.detach().to(torch.float64).cpu().numpy()


def some(sizes, dtypes, scale=0.1, seed=1):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return [(torch.randn(n, generator=g, device="cuda") * scale).to(DTYPES[dtypes[i % len(dtypes)]]) for i, n in enumerate(sizes)]


def truth(grads):
    return math.sqrt(math.fsum(float((host(g).ravel() ** 2).sum()) for g in grads))


def check(grads, max_norm, out=None):
    """Norm to one fp32 rounding (the fp64 sums' own error is far below it),
    scaled values to the factor's, the product's and the result's rounding."""
    before = [host(g) for g in grads]
    want = truth(grads)
    alone = lt().grad_norm(grads)
    norm = lt().clip_grad_norm(grads, max_norm, out=out)
    assert norm.dtype == torch.float32 and norm.shape == () and norm.is_cuda
    assert abs(float(norm) - want) <= 1.01 * 2.0 ** -24 * want and float(alone) == float(norm)
    c = 1.0 if want <= max_norm else max_norm / want
    for g, b, o in zip(grads, before, grads if out is None else out):
        u = UNIT[str(g.dtype).split(".")[1]]
        got = host(o)
        assert np.all(np.abs(got - c * b) <= (2.02 * 2.0 ** -24 + u) * np.abs(c * b) + (2.0 ** -24 if u == 2.0 ** -11 else 2.0 ** -133))
        if out is not None:
            assert np.array_equal(host(g), b)
        if c == 1.0:
            assert np.array_equal(got, b)


@pytest.mark.parametrize("dtypes", [("float32",), ("bfloat16",), ("float16",), ("float32", "bfloat16", "float16")])
@pytest.mark.parametrize("sizes", [[1], [7, 0, 300], [8192, 16384, 16385, 3], [1_000_003], list(range(1, 400)),
                                   [50_000 + 37 * i for i in range(130)], [0, 0, 5]])
@pytest.mark.parametrize("into", [False, True])
def test_clip(sizes, dtypes, into):
    print(f"[clip] {len(sizes)} tensors {dtypes} into {into}", flush=True)
    grads = some(sizes, dtypes)
    out = [torch.full_like(g, 7.0) for g in grads] if into else None
    check(grads, 0.05, out)


@pytest.mark.parametrize("into", [False, True])
def test_below_the_limit(into):
    grads = some([1000, 77], ["float32", "bfloat16"])
    check(grads, 1e6, [torch.full_like(g, 7.0) for g in grads] if into else None)


def test_unaligned_and_shapes():
    base = some([40_000], ["bfloat16"])[0]
    grads = [base[1:9000], base[9001:9004], base[20_003:39_999], torch.randn(33, 65, device="cuda").t(),
             torch.randn(3, 5, 7, device="cuda").permute(2, 0, 1), torch.randn((), device="cuda")]
    check(grads, 0.25, [torch.empty_strided(g.shape, g.stride(), dtype=g.dtype, device="cuda") for g in grads])


@pytest.mark.parametrize("scale", [1e30, 1e-30, 1e-38])
def test_magnitudes(scale):
    check(some([5000, 129], ["float32"], scale), 1.0)


def test_zero_and_empty():
    z = torch.zeros(100, device="cuda")
    assert float(lt().clip_grad_norm([z], 1.0)) == 0.0 and not host(z).any()
    assert float(lt().clip_grad_norm([z], 0.0)) == 0.0 and not host(z).any()
    e = torch.zeros(0, device="cuda")
    assert float(lt().grad_norm([e, e])) == 0.0 and float(lt().clip_grad_norm([e], 1.0)) == 0.0


def test_clip_to_zero():
    g = torch.ones(100, device="cuda")
    assert float(lt().clip_grad_norm([g], 0.0)) == 10.0 and not host(g).any()


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_not_finite(bad):
    """The formula: an infinite norm scales by zero, a NaN norm by NaN."""
    g = torch.ones(20_000, device="cuda")
    g[12_345] = bad
    norm = float(lt().clip_grad_norm([g], 1.0))
    h = host(g)
    if math.isnan(bad):
        assert math.isnan(norm) and np.isnan(h).all()
    else:
        assert norm == math.inf and np.isnan(h[12_345]) and not np.delete(h, 12_345).any()


def test_reproducible():
    grads = some([333_333, 1, 70_001], ["float32", "float16"])
    assert len({float(lt().grad_norm(grads)) for _ in range(5)}) == 1


def test_the_same_tensor_twice():
    """Counted twice in a norm; refused where it would be scaled twice at once."""
    g = torch.full((8,), 2.0, device="cuda")
    e = torch.zeros(0, device="cuda")
    assert float(lt().grad_norm([g, g])) == 8.0
    with pytest.raises(ValueError):
        lt().clip_grad_norm([g, e, e, g], 1.0)
    out = [torch.empty_like(g), e, e, torch.empty_like(g)]
    assert float(lt().clip_grad_norm([g, e, e, g], 4.0, out=out)) == 8.0
    assert (out[0] == 1.0).all() and (out[3] == 1.0).all() and (g == 2.0).all()

"""Clipping where the norm or the factor leaves the range of fp32 and the scaled
gradients do not."""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

from test_gpu_grad_clip import DTYPES, UNIT, host, lt

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("max_norm", [1e3, 1.0, 1e-3, 1e-7, 1e-20])
@pytest.mark.parametrize("size", [1e38, 3e36, 1e30])
@pytest.mark.parametrize("into", [False, True])
def test_small_factors(into, size, max_norm, dtype):
    """Factors down to 1e-60: rounded to fp32's precision, the product and the result
    rounded once each; below the normal range one spacing."""
    g = torch.Generator(device="cuda").manual_seed(3)
    v = ((torch.rand(1003, generator=g, device="cuda") + 0.5) * size).to(DTYPES[dtype])
    v[::2] *= -1
    b = host(v)
    want = math.sqrt(math.fsum(b * b))
    out = [torch.empty_like(v)] if into else None
    norm = float(lt().clip_grad_norm([v], max_norm, out=out))
    with np.errstate(over="ignore"):
        assert norm == float(np.float32(want)) or abs(norm - want) <= 2.0 ** -23 * want
    got, c = host(out[0] if into else v), max_norm / want
    spacing = 2.0 ** -149 if dtype == "float32" else 2.0 ** -133
    assert (np.abs(got - c * b) <= (2.02 * 2.0 ** -24 + UNIT[dtype]) * np.abs(c * b) + spacing).all()
    if max_norm > 1e-20:
        assert got.all()


def test_infinite_norm_of_finite_gradients():
    """A norm above fp32's range is returned as infinity and scales by its value."""
    v = torch.full((100,), 1e38, device="cuda")
    assert float(lt().grad_norm([v])) == math.inf
    assert float(lt().clip_grad_norm([v], 1.0)) == math.inf
    assert np.abs(host(v) - 0.1).max() <= 0.1 * 2.0 ** -22

"""Group norm's mean and rstd: rounded about once, also where a rounding of theirs decides
on which side of relu's border a value lies."""
from __future__ import annotations

import pytest
import torch

pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.bfloat16, torch.float16]
# (c, s, b), groups: in a workgroup's registers (one group a vector, several, vectors that are not
# whole, a few channels), and the features of tokens in a wave and in a workgroup
ONE_READ = [((6, 5, 3), 2), ((3, 35, 2), 3), ((90, 45, 7), 9), ((256, 729, 2), 32), ((64, 169, 3), 32), ((40, 16, 65), 4), ((1000, 1, 41), 8),
            ((4001, 1, 5), 1), ((8192, 1, 3), 1)]


def lt():
    import paper_2005_06410_amd as m
    return m


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def stored(v, dtype):
    """(c, s, b) values with the channels fastest."""
    return v.permute(2, 1, 0).contiguous().to(dtype).permute(2, 1, 0)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape,groups", ONE_READ)
def test_mean_is_rounded_once(shape, groups, dtype):
    """Whole numbers below 16: their sums are exact in fp32 (n 15 < 2^24), and the mean is the
    quotient's one rounding."""
    c, s, b = shape
    x = stored(torch.randint(0, 16, shape, generator=gen(c + s), device="cuda"), dtype)
    _, mean, _ = lt().group_norm(x, groups)
    n = c // groups * s
    want = x.double().reshape(groups, n, b).sum(1) / n
    assert torch.equal(mean, want.float())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape,groups", ONE_READ)
def test_rstd_is_rounded_once(shape, groups, dtype):
    """Whole numbers that lie evenly around 3: mean, differences and squares are exact, and so
    is eps.  The quotient, the sum and the step keep what their roundings lose but for second
    orders (2^-44 in all), the last sum is rounded once: 2^-24 (1 + 2^-16) of rstd."""
    c, s, b = shape
    n = c // groups * s
    half = torch.randint(-7, 8, (groups, n // 2, b), generator=gen(c + s), device="cuda")
    e = torch.cat([half, torch.zeros((groups, n % 2, b), device="cuda", dtype=half.dtype), -half], 1)
    x = stored(3 + e.reshape(shape), dtype)
    eps = 2.0 ** -10
    _, mean, rstd = lt().group_norm(x, groups, eps=eps)
    assert (mean == 3).all()
    want = ((e.double() ** 2).sum(1) / n + eps) ** -0.5
    off = (rstd.double() / want - 1).abs()
    assert (off <= 2.0 ** -24 * (1 + 2.0 ** -16)).all(), float(off.max()) * 2.0 ** 24


def test_rstd_without_variance():
    """Where the variance is 0, rstd is 1 / sqrt(eps), and infinite where eps is 0 too."""
    x = stored(torch.full((8, 9, 2), 3.0, device="cuda"), torch.float32)
    for eps in (0.0, 2.0 ** -10, 2.0 ** -100):
        _, mean, rstd = lt().group_norm(x, 2, eps=eps)
        want = torch.tensor(eps, dtype=torch.float64, device="cuda") ** -0.5
        assert (mean == 3).all() and (rstd.double() == want).all()


# (c, s, b), groups, and the values of a channel that a thread takes at the most
CHUNKED = [((32, 25600, 1), 8, 4), ((16, 1 << 19, 2), 4, 16), ((16, (1 << 24) - 1, 1), 4, 64), ((4, 65536, 4100), 1, 256)]


@pytest.mark.parametrize("far", [200.0, 12345.678, 1e6])
@pytest.mark.parametrize("base", [None, 0.1])
@pytest.mark.parametrize("shape,groups,held", CHUNKED)
def test_a_far_first_value(shape, groups, held, base, far):
    """Large maps in chunks whose first position holds a value far from all others, which are
    normal or all the same: most of the variance is that value's, and what the thread that met
    it first makes of it shows whole.

    In units of 2^-24 of the sum of squares: four values' squares and their sum's square are off by
    20 of the squares, of which a quarter or more stays: 80; what a thread adds up, one each
    of held / 4 steps; its mean is off by two of the far value a step, which enters the
    squares around the chunk's mean twice: together 5 a step, 5 / 4 held; the others' differences, which are
    rounded at the far value's size, at most 16; the sums over threads, chunks and channels
    pass at most 64 additions.  rstd is off by half of all this and its own rounding.  The
    mean: 64 additions of the values' size, and in the threads that begin with the far value
    two roundings of it a step."""
    c, s, b = shape
    n = c // groups * s
    x = torch.empty((b, s, c), device="cuda")
    if base is None:
        x.normal_(generator=gen(c))
    else:
        x.fill_(base)
    x[:, 0] = far
    _, mean, rstd = lt().group_norm(x.permute(2, 1, 0), groups, eps=2.0 ** -20)
    for image in {0, b - 1}:
        v = x[image].double().reshape(s, groups, c // groups)
        m = v.mean((0, 2))
        want = ((v - m[:, None]) ** 2).mean((0, 2)).add(2.0 ** -20) ** -0.5
        off = (rstd[:, image].double() / want - 1).abs()
        bound = (160 + 5 * held / 4) / 2 * 2.0 ** -24 + 2.0 ** -24
        assert (off <= bound).all(), f"rstd is off by {float(off.max()):.3g}, {float(off.max()) / bound:.3g} times its bound"
        size = v.abs().mean((0, 2))
        assert ((mean[:, image].double() - m).abs() <= 2.0 ** -24 * (64 * size + far * held * held / 2 / s)).all()


@pytest.mark.parametrize("shape,groups", [((0, 4, 3), 1), ((8, 0, 5), 4), ((8, 0, 300000), 2), ((8, 4, 0), 2)])
def test_statistics_of_nothing(shape, groups):
    """Images without a value have the mean 0 / 0; without images there is nothing to write."""
    c, s, b = shape
    size = (1, c, s, b, groups)
    apart = (max(c, 1), max(c, 1) * max(s, 1))
    stream = torch.cuda.current_stream().cuda_stream
    for which in ((0, 1), (0,), (1,), ()):
        held = torch.full((2, groups * b + 8), 5.0, device="cuda")
        at = [held[i].data_ptr() if i in which else 0 for i in range(2)]
        assert lt().load().convgemm_group_norm(*size, 0, *apart, 0, 0, 1e-5, 0, 0, *apart, *at, 0, 0, stream) == 0
        for i in range(2):
            written = groups * b if i in which else 0
            assert held[i, :written].isnan().all() and (held[i, written:] == 5).all()
    x = torch.empty((b, s, c), device="cuda").permute(2, 1, 0)
    _, mean, rstd = lt().group_norm(x, groups)
    assert mean.shape == rstd.shape == (groups, b) and mean.isnan().all() and rstd.isnan().all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape,groups", ONE_READ + [((30, 22650, 2), 5), ((7, 20011, 2), 7), ((12, 40000, 1), 1)])
def test_gradients_of_scaled_inputs(shape, groups, dtype):
    """Inputs of 2^-k times the size, and rstd 2^k times as large: dI is 2^k times as large and
    the others are the same, bit for bit, since nothing is rounded differently."""
    c, s, b = shape
    g = gen(c + s)
    x, dO = (stored(torch.randn(shape, generator=g, device="cuda"), dtype) for _ in range(2))
    w, bias = ((at + 0.3 * torch.randn(c, generator=g, device="cuda")).to(dtype) for at in (1, 0))
    _, mean, rstd = lt().group_norm(x, groups, w, bias)
    want = lt().group_norm_backward(x, dO, groups, mean, rstd, w, bias, activation="silu")
    for k in (-60, 50, 66, 90):
        got = lt().group_norm_backward(x * 2.0 ** -k, dO, groups, mean * 2.0 ** -k, rstd * 2.0 ** k, w, bias, activation="silu")
        # what is near bf16's or fp32's smallest values is rounded there
        assert torch.equal(torch.where(want[0].abs() < 2.0 ** -60, 0, got[0]), torch.where(want[0].abs() < 2.0 ** -60, 0, want[0]) * 2.0 ** k)
        assert torch.equal(got[1], want[1]) and torch.equal(got[2], want[2])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape,groups", ONE_READ)
def test_squares_and_sums_beyond_the_range(shape, groups, dtype):
    """Squares that leave fp32's range make rstd 0 and O the bias; a sum that does makes the mean
    infinite."""
    c, s, b = shape
    n = c // groups * s
    sign = (torch.arange(n, device="cuda") % 2 * 2 - 1.0) * (torch.arange(n, device="cuda") < n // 2 * 2)
    x = stored((sign * 1e20)[None, :, None].expand(groups, n, b).reshape(shape), dtype)
    bias = torch.randn(c, generator=gen(c), device="cuda").to(dtype)
    o, mean, rstd = lt().group_norm(x, groups, bias=bias)
    assert (mean == 0).all() and (rstd == 0).all() and torch.equal(o, bias[:, None, None].expand(shape))
    _, mean, _ = lt().group_norm(stored(torch.full(shape, 3e38, device="cuda"), dtype), groups)
    assert (mean == torch.inf).all()

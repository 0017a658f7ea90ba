"""Group norm with an activation and its gradients against their 64-bit forms, at the
sizes, groupings, strides and values where they can go wrong."""
from __future__ import annotations

import pytest
import torch

import norm_truths as truth

pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.bfloat16, torch.float16]
ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]


def lt():
    import paper_2005_06410_amd as m
    return m


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def maps(g, shape, dtype, pad=0, gap=0, shift=0, offset=1.0):
    """(c, ..., b) values, channels fastest: `pad` values behind each position, `gap`
    behind each image, `shift` into the buffer; every channel with an offset."""
    c, b, s = shape[0], shape[-1], 1
    for n in shape[1:-1]:
        s *= n
    ld = c + pad
    ldb = s * ld + gap
    flat = torch.full((shift + b * ldb + 8,), 9.0, dtype=dtype, device="cuda")
    strides = [1]
    for n in shape[1:-1]:
        strides.append(ld)
        ld *= n
    v = flat.as_strided(shape, tuple(strides) + (ldb,), shift)
    offsets = torch.randn((c,) + (1,) * (len(shape) - 1), generator=g, device="cuda") * offset
    v.copy_(torch.randn(shape, generator=g, device="cuda") + offsets)
    return v


def flat3(v):
    return v.reshape(v.shape[0], -1, v.shape[-1])


def within(got, want, bound, what):
    off = (got.double() - want).abs()
    bad = ~(off <= bound)
    if got.dtype == torch.float16:
        # fp16's largest value is (2 - 2^-10) 2^15, and what lies half a step above it,
        # (2 - 2^-11) 2^15 = 65520, or beyond rounds to infinity: the rounding of a result
        # whose error reaches that far
        bad &= ~(got.isinf() & (got.double().sign() == want.sign()) & (want.abs() + bound >= 65520))
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, the worst {float((off / bound)[bad].max()):.3g} times its bound"


def check(x, dO, groups, w, b, act, eps=1e-5):
    o, mean, rstd = lt().group_norm(x, groups, w, b, eps=eps, activation=act)
    dI, dw, db = lt().group_norm_backward(x, dO, groups, mean, rstd, w, b, activation=act)
    x3, d3 = flat3(x), flat3(dO)
    want = truth.norm(x3, groups, w, b, eps, act)[:3] + truth.backward(x3, d3, groups, w, b, eps, act)
    bound = truth.bounds(x3, groups, w, b, eps, act, d3)
    assert o.shape == dI.shape == x.shape and o.dtype == dI.dtype == dw.dtype == db.dtype == x.dtype
    for got, v, e, what in zip((flat3(o), mean, rstd, flat3(dI), dw, db), want, bound, ("O", "mean", "rstd", "dI", "dweight", "dbias")):
        within(got, v, e, what)
    return o, mean, rstd, dI, dw, db


def affine(g, c, dtype):
    return (1 + 0.3 * torch.randn(c, generator=g, device="cuda")).to(dtype), (0.3 * torch.randn(c, generator=g, device="cuda")).to(dtype)


# (shape, groups): one value; one channel a group; groups of every width next to the vectors'; units of
# several groups; maps smaller than a workgroup; one group; maps in chunks, also of a few channels or of thousands
SIZES = [((1, 1), 1), ((6, 5, 3), 2), ((3, 7, 5, 2), 3), ((90, 9, 5, 7), 9), ((64, 13, 13, 3), 32), ((384, 13, 13, 1), 32), ((256, 27, 27, 4), 32),
         ((1000, 41), 8), ((40, 4, 4, 65), 4), ((128, 64, 64, 2), 32), ((24, 300, 2), 1), ((12, 150, 150, 1), 4), ((7, 20011, 2), 7),
         ((1, 70001, 1), 1), ((2048, 2, 3, 5), 1), ((9000, 3, 2), 3), ((4100, 30, 2), 2), ((20000, 1, 3), 1), ((520, 1, 700), 65), ((16, 40000, 3), 16), ((3, 5000), 1), ((4, 3001), 2),
         ((264, 999), 3), ((4096, 70), 2), ((530, 33), 5), ((1024, 77), 1)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape,groups", SIZES)
def test_sizes(shape, groups, dtype):
    g = gen(sum(shape))
    x, dO = maps(g, shape, dtype), maps(g, shape, dtype, offset=0.1)
    w, b = affine(g, shape[0], dtype)
    act = ACTS[sum(shape) % 5]
    check(x, dO, groups, w, b, act)


# groups of more features than a wave holds, also not whole vectors and of more tokens than
# workgroups; groups whose chunks are joined by channel first
WIDE = [((1100, 5), 1), ((2060, 9), 2), ((2052, 3), 1), ((8192, 3), 1), ((4097, 700), 1), ((16384, 2), 1), ((16390, 3), 1), ((9001, 600), 1), ((12300, 1), 2),
        ((2000, 40, 40, 1), 1), ((515, 70, 70, 2), 1), ((1030, 50, 50, 1), 2), ((6000, 130, 2), 1)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape,groups", WIDE)
def test_wide_groups(shape, groups, dtype):
    g = gen(sum(shape))
    x, dO = maps(g, shape, dtype), maps(g, shape, dtype, offset=0.1)
    w, b = affine(g, shape[0], dtype)
    _, mean, rstd, dI, dw, db = check(x, dO, groups, w, b, ACTS[sum(shape) % 5])
    # what is left out changes nothing in what is not
    act = ACTS[sum(shape) % 5]
    for needs in [(1, 0, 0), (0, 1, 1)]:
        for need, got, v in zip(needs, lt().group_norm_backward(x, dO, groups, mean, rstd, w, b, activation=act, needs=needs), (dI, dw, db)):
            assert got is None if not need else torch.equal(got, v)
    # in place
    want = lt().group_norm(x, groups, w, b, activation=act)[0]
    assert torch.equal(lt().group_norm(x, groups, w, b, activation=act, out=x)[0], want)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", DTYPES)
def test_activations(dtype, act):
    g = gen(3)
    for shape, groups in [((48, 11, 5, 3), 6), ((32, 130, 130, 1), 8)]:
        x, dO = maps(g, shape, dtype), maps(g, shape, dtype)
        w, b = affine(g, shape[0], dtype)
        check(x, dO, groups, w, b, act)
        check(x, dO, groups, w, None, act)
        check(x, dO, groups, None, b, act)


@pytest.mark.parametrize("pad,gap,shift", [(8, 0, 0), (3, 5, 0), (0, 0, 1), (5, 16, 3)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_strides_and_addresses(dtype, pad, gap, shift):
    g = gen(pad + gap + shift)
    for shape, groups in [((96, 6, 7, 5), 8), ((30, 150, 151, 2), 5)]:
        x, dO = maps(g, shape, dtype, pad, gap, shift), maps(g, shape, dtype, gap, pad, shift)
        w, b = affine(g, shape[0], dtype)
        check(x, dO, groups, w, b, "silu")
        out = maps(g, shape, dtype, pad, gap, shift)
        behind = out.clone()
        lt().group_norm(x, groups, w, b, activation="silu", out=out)
        assert torch.equal(out, lt().group_norm(x, groups, w, b, activation="silu")[0]) and not torch.equal(out, behind)
        # what lies between the positions stays
        whole = out.as_strided((shape[-1] * out.stride(-1) - gap,), (1,), out.storage_offset())
        if pad:
            rest = whole.as_strided((shape[1] * shape[2], pad), (shape[0] + pad, 1), out.storage_offset() + shape[0])
            assert (rest == 9).all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_in_place(dtype):
    g = gen(5)
    for shape, groups in [((96, 6, 7, 5), 8), ((30, 150, 151, 2), 5)]:
        x = maps(g, shape, dtype)
        w, b = affine(g, shape[0], dtype)
        want = lt().group_norm(x, groups, w, b, activation="relu")
        y = x.clone(memory_format=torch.preserve_format)
        got = lt().group_norm(y, groups, w, b, activation="relu", out=y)
        assert got[0] is y
        for a, v in zip(got, want):
            assert torch.equal(a, v)


@pytest.mark.parametrize("dtype", DTYPES)
def test_values_far_from_zero(dtype):
    """A mean thousands of deviations from zero, and a first value far from the others:
    the squares are summed around the mean."""
    g = gen(6)
    for shape, groups in [((32, 9, 9, 3), 8), ((32, 160, 160, 1), 8)]:
        for offset, outlier in ((512.0, 0.0), (0.0, 200.0)):
            x = maps(g, shape, dtype, offset=0.0)
            x += offset
            if dtype != torch.float32 and offset:
                x.copy_((x.float() - offset).round() * 8 + offset)
            x[:, 0, 0] += outlier
            dO = maps(g, shape, dtype)
            w, b = affine(g, shape[0], dtype)
            check(x, dO, groups, w, b, "gelu")


def test_constant_groups():
    """No variance: xhat is 0 and O is act(bias); eps bounds rstd."""
    g = gen(7)
    for s in (9, 30000):
        x = torch.full((16, s, 2), 3.0, device="cuda").permute(2, 1, 0).contiguous().permute(2, 1, 0)
        w, b = affine(g, 16, torch.float32)
        o, mean, rstd = lt().group_norm(x, 4, w, b)
        assert (mean == 3).all() and torch.equal(o, b[:, None, None].expand_as(o))
        # eps is rounded to fp32 (half of it remains under the root), the root and the
        # quotient are rounded once each
        want = torch.full_like(rstd, 1e-5 ** -0.5, dtype=torch.float64)
        within(rstd, want, 3 * 2.0 ** -24 * want, "rstd")


@pytest.mark.parametrize("dtype", DTYPES)
def test_infinities_stay_in_their_group(dtype):
    g = gen(8)
    for shape, groups in [((36, 5, 5, 4), 6), ((36, 140, 150, 2), 6)]:
        x, dO = maps(g, shape, dtype), maps(g, shape, dtype)
        w, b = affine(g, shape[0], dtype)
        clean = lt().group_norm(x, groups, w, b, activation="silu")
        cleand = lt().group_norm_backward(x, dO, groups, clean[1], clean[2], w, b, activation="silu")
        per = shape[0] // groups
        for bad in (torch.inf, torch.nan):
            y = x.clone(memory_format=torch.preserve_format)
            y[per + 1, 2, 3, 1] = bad
            o, mean, rstd = lt().group_norm(y, groups, w, b, activation="silu")
            dI, dw, db = lt().group_norm_backward(y, dO, groups, mean, rstd, w, b, activation="silu")
            hit = torch.zeros(groups, shape[-1], dtype=torch.bool, device="cuda")
            hit[1, 1] = True
            where = hit.repeat_interleave(per, 0)[:, None, None, :].expand(shape)
            assert o[where].isnan().all() and dI[where].isnan().all()
            assert torch.equal(o[~where], clean[0][~where]) and torch.equal(dI[~where], cleand[0][~where])
            assert dw[per:2 * per].isnan().all()
            keep = [i for i in range(shape[0]) if not per <= i < 2 * per]
            assert torch.equal(dw[keep], cleand[1][keep]) and torch.equal(db[keep], cleand[2][keep])


def test_gradients_are_differences():
    """Central differences of the definition along random directions."""
    g = gen(9)
    for shape, groups in [((24, 4, 5, 3), 4), ((8, 170, 170, 1), 2)]:
        x, dO = maps(g, shape, torch.float32), maps(g, shape, torch.float32)
        w, b = affine(g, shape[0], torch.float32)
        _, mean, rstd = lt().group_norm(x, groups, w, b, activation="silu")
        grads = lt().group_norm_backward(x, dO, groups, mean, rstd, w, b, activation="silu")
        h = 2.0 ** -10
        for i, got in enumerate(grads):
            args = [x.double(), w.double(), b.double()]
            d = torch.randn(args[i].shape, generator=g, device="cuda", dtype=torch.float64)
            values = []
            for sign in (1, -1):
                moved = list(args)
                moved[i] = args[i] + sign * h * d
                values.append((truth.norm(flat3(moved[0]), groups, moved[1], moved[2], 1e-5, "silu")[0] * flat3(dO).double()).sum())
            want = float((values[0] - values[1]) / (2 * h))
            slope = float((got.double() * d).sum())
            assert abs(slope - want) <= 1e-4 * (abs(want) + float((got.double() * d).norm())), (i, slope, want)


@pytest.mark.parametrize("dtype", DTYPES)
def test_outputs_that_are_left_out(dtype):
    g = gen(10)
    for shape, groups in [((40, 5, 6, 7), 5), ((24, 170, 170, 1), 3)]:
        x, dO = maps(g, shape, dtype), maps(g, shape, dtype)
        w, b = affine(g, shape[0], dtype)
        _, mean, rstd = lt().group_norm(x, groups, w, b, activation="gelu")
        every = lt().group_norm_backward(x, dO, groups, mean, rstd, w, b, activation="gelu")
        for needs in [(1, 0, 0), (0, 1, 0), (0, 0, 1), (0, 1, 1), (1, 1, 0), (0, 0, 0)]:
            got = lt().group_norm_backward(x, dO, groups, mean, rstd, w, b, activation="gelu", needs=needs)
            for n, a, v in zip(needs, got, every):
                assert (a is None) == (not n)
                if n:
                    assert torch.equal(a, v)


def test_empty_extents():
    for shape in [(0, 4, 4, 2), (8, 0, 4, 2), (8, 4, 4, 0)]:
        x = torch.empty(tuple(reversed(shape)), device="cuda").permute(3, 2, 1, 0)
        w = torch.ones(shape[0], device="cuda")
        o, mean, rstd = lt().group_norm(x, 1, w, w)
        assert o.shape == shape and mean.shape == (1, shape[3])
        dI, dw, db = lt().group_norm_backward(x, x, 1, mean, rstd, w, w)
        assert dI.shape == shape and not dw.any() and not db.any()


def test_workspace_is_not_left():
    """The C call with exactly the bytes that the query names, in a buffer whose other
    values stay."""
    import ctypes
    m = lt()
    lib = m.load()
    g = gen(11)
    for shape, groups in [((96, 6, 7, 5), 8), ((30, 150, 151, 2), 5), ((7, 20011, 2), 7), ((9000, 3, 2), 3)]:
        x, dO = maps(g, shape, torch.bfloat16), maps(g, shape, torch.bfloat16)
        c, b = shape[0], shape[-1]
        s = x.numel() // c // b
        o, mean, rstd = m.group_norm(x, groups)
        dI = torch.empty_like(x)
        dw, db = torch.empty(c, dtype=x.dtype, device="cuda"), torch.empty(c, dtype=x.dtype, device="cuda")
        size = (4, c, s, b, groups)
        maps_ = (c, c * s)
        for back in (0, 1):
            need = (lib.convgemm_group_norm_backward_workspace if back else lib.convgemm_group_norm_workspace)(*size)
            buffer = torch.full((need + 512,), 77, dtype=torch.uint8, device="cuda")
            ws = buffer.data_ptr() + 256
            stream = torch.cuda.current_stream().cuda_stream
            if back:
                code = lib.convgemm_group_norm_backward(*size, x.data_ptr(), *maps_, dO.data_ptr(), *maps_, 0, 0, 4, mean.data_ptr(), rstd.data_ptr(),
                                                        dI.data_ptr(), *maps_, dw.data_ptr(), db.data_ptr(), ws, need, stream)
            else:
                code = lib.convgemm_group_norm(*size, x.data_ptr(), *maps_, 0, 0, ctypes.c_double(1e-5), 4, o.data_ptr(), *maps_, mean.data_ptr(),
                                               rstd.data_ptr(), ws, need, stream)
            assert code == 0
            assert (buffer[:256] == 77).all() and (buffer[256 + need:] == 77).all()


def test_maps_beyond_32_bit_offsets():
    """More than 2^31 values, in one image and over images: rows of 1 and -1 in turn have
    the mean 0 (or 1 / s of a row) and the variance 1."""
    for c, s, b in [(256, (1 << 23) + 4, 1), (64, 1 << 20, 34)]:
        sign = (torch.arange(s, device="cuda", dtype=torch.int32) % 2 * 2 - 1).to(torch.bfloat16)
        x = sign[:, None].expand(b, s, c).contiguous().permute(2, 1, 0)
        assert x.numel() > 1 << 31
        o, mean, rstd = lt().group_norm(x, 8, eps=3.0)
        assert (mean.abs() < 1e-6).all() and ((rstd - 0.5).abs() < 1e-6).all()
        for p in (slice(0, 1000), slice(s - 1000, s)):
            assert torch.equal(o[:, p, b - 1], x[:, p, b - 1] / 2)
        del o
        # dO of ones: d - avg d = 0, and xhat has no part in it
        one = torch.ones((), dtype=torch.bfloat16, device="cuda").expand(b, s, c).contiguous().permute(2, 1, 0)
        dI, dw, db = lt().group_norm_backward(x, one, 8, mean, rstd)
        for p in (slice(0, 1000), slice(s - 1000, s)):
            assert (dI[:, p, b - 1].float().abs() < 1e-6).all()
        assert ((db.float() - b * s).abs() <= 2.0 ** -8 * b * s).all()
        del x, one, dI


def test_streams_graphs_and_repeats():
    g = gen(12)
    cases = []
    for shape, groups, dtype in [((64, 12, 12, 9), 8, torch.bfloat16), ((24, 170, 170, 2), 3, torch.float16)]:
        cases.append((maps(g, shape, dtype), maps(g, shape, dtype), groups) + affine(g, shape[0], dtype))

    def step(c):
        x, dO, groups, w, b = c
        o, mean, rstd = lt().group_norm(x, groups, w, b, activation="silu")
        return (o, mean, rstd) + lt().group_norm_backward(x, dO, groups, mean, rstd, w, b, activation="silu")

    want = [step(c) for c in cases]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = [step(c) for c in cases]
    torch.cuda.current_stream().wait_stream(side)
    graphs, held = [], []
    for c in cases:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            held.append(step(c))
        graphs.append(graph)
    for _ in range(3):
        for graph in graphs:
            graph.replay()
        again = [step(c) for c in cases]
        torch.cuda.synchronize()
        for w, h, a, o in zip(want, held, again, other):
            for x, y, z, v in zip(w, h, a, o):
                assert torch.equal(x, y) and torch.equal(x, z) and torch.equal(x, v)
        for h in held:
            for v in h:
                v.zero_()


def test_refusals():
    g = gen(13)
    x = maps(g, (24, 5, 6, 2), torch.bfloat16)
    w, b = affine(g, 24, torch.bfloat16)
    m = lt()
    o, mean, rstd = m.group_norm(x, 4, w, b)
    row = x.contiguous()
    bad = [
        (ValueError, lambda: m.group_norm(row, 4)),
        (ValueError, lambda: m.group_norm(x, 5)),
        (ValueError, lambda: m.group_norm(x, 0)),
        (ValueError, lambda: m.group_norm(x.cpu(), 4)),
        (ValueError, lambda: m.group_norm(x[:, 0, 0, 0], 4)),
        (ValueError, lambda: m.group_norm(x[:, :4], 4)),
        (ValueError, lambda: m.group_norm(x, 4, w[:23])),
        (TypeError, lambda: m.group_norm(x, 4, w.float())),
        (TypeError, lambda: m.group_norm(x.double(), 4)),
        (ValueError, lambda: m.group_norm(x, 4, w, b, eps=-1.0)),
        (ValueError, lambda: m.group_norm(x, 4, w, b, eps=float("nan"))),
        (ValueError, lambda: m.group_norm(x, 4, w, b, activation="tanh")),
        (ValueError, lambda: m.group_norm(x, 4, w, b, out=x[..., :1])),
        (TypeError, lambda: m.group_norm(x, 4, w, b, out=torch.empty_like(x, dtype=torch.float16))),
        (ValueError, lambda: m.group_norm(x[..., :1], 4, out=x.as_strided((24, 5, 6, 1), x.stride(), x.storage_offset() + 24))),
        (ValueError, lambda: m.group_norm_backward(x, row, 4, mean, rstd, w, b)),
        (TypeError, lambda: m.group_norm_backward(x, o.float(), 4, mean, rstd, w, b)),
        (ValueError, lambda: m.group_norm_backward(x, o, 4, mean[:3], rstd, w, b)),
        (ValueError, lambda: m.group_norm_backward(x, o, 4, mean.contiguous(), rstd, w, b)),
        (TypeError, lambda: m.group_norm_backward(x, o, 4, mean.half(), rstd, w, b)),
    ]
    for error, call in bad:
        with pytest.raises(error):
            call()

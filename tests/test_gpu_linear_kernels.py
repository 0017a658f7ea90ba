"""Every kernel of the layer's product, with operands in every order, aligned and
not, on sums of small integers: exact in any order of summation and in every
type, so results must equal the 64-bit product's bit for bit.  The sizes are
those at which the library takes each kernel; operands above 4 GiB come last."""
from __future__ import annotations

import pytest
import torch

pytestmark = pytest.mark.gpu

# (weights' order, kernel's number, kn, ci, t): order 1 = ci fastest
WIDE_TYPES = [  # bfloat16 and float16
    (0, 0, 5752, 336, 1469), (0, 1, 3760, 80, 1156), (0, 2, 3840, 96, 514), (0, 2, 8776, 2864, 106), (0, 3, 1560, 336, 2443),
    (0, 4, 2360, 96, 1), (0, 4, 184, 2760, 2), (0, 5, 8776, 640, 28), (0, 5, 744, 2184, 340), (0, 6, 184, 1200, 1),
    (0, 6, 872, 2856, 23), (0, 7, 8520, 400, 19), (0, 8, 6280, 208, 4), (0, 8, 808, 2832, 34),
    (1, 0, 6560, 344, 1326), (1, 1, 2144, 72, 2181), (1, 2, 8952, 80, 206), (1, 2, 2056, 2680, 460), (1, 3, 6680, 288, 535),
    (1, 4, 872, 144, 1), (1, 4, 48, 2976, 80), (1, 5, 8560, 616, 17), (1, 5, 1040, 2496, 238), (1, 6, 2048, 176, 1),
    (1, 6, 288, 3088, 100), (1, 7, 8536, 472, 22), (1, 8, 7912, 368, 1), (1, 9, 104, 2192, 1)]
SINGLE = [
    (0, 1, 3248, 104, 2058), (0, 10, 1072, 416, 295), (0, 10, 2328, 2224, 72), (0, 11, 416, 176, 123), (0, 11, 208, 3136, 72),
    (0, 2, 1272, 80, 2455), (0, 2, 4200, 928, 244), (0, 3, 2320, 408, 386), (0, 3, 1568, 1584, 343), (0, 4, 1216, 72, 336),
    (0, 4, 104, 1400, 1), (0, 5, 768, 448, 462), (0, 5, 160, 1672, 931), (0, 6, 176, 152, 810), (0, 6, 2696, 1888, 19),
    (0, 7, 9032, 104, 18), (0, 7, 2840, 1312, 19), (0, 8, 128, 72, 3), (0, 8, 128, 1936, 1),
    (1, 1, 5432, 80, 1237), (1, 10, 3088, 296, 140), (1, 10, 2400, 2304, 67), (1, 11, 128, 128, 283), (1, 11, 216, 704, 280),
    (1, 2, 4000, 72, 780), (1, 2, 2416, 1040, 448), (1, 3, 832, 392, 1229), (1, 3, 4712, 1424, 101), (1, 4, 1848, 88, 162),
    (1, 4, 224, 1376, 95), (1, 5, 472, 440, 704), (1, 5, 216, 1672, 762), (1, 6, 112, 120, 1205), (1, 6, 2720, 2304, 32),
    (1, 7, 5608, 72, 34), (1, 7, 2336, 1944, 20), (1, 8, 1088, 128, 1), (1, 8, 400, 2040, 3), (1, 9, 208, 320, 1),
    (1, 9, 112, 1872, 1)]
CASES = [(d, *c) for d in (torch.bfloat16, torch.float16) for c in WIDE_TYPES] + [(torch.float32, *c) for c in SINGLE]


def lt():
    import paper_2005_06410_amd as m
    return m


def ints(gen, shape, density, dtype, shift=0, pad=0, order=0):
    """-1, 0, 1 of the given density, first index fastest (order 0) or last; NaN
    in the gaps of a padded or shifted tensor."""
    rows, cols = shape if order == 0 else shape[::-1]
    v = torch.randint(0, 3, (cols, rows), generator=gen, device="cuda") - 1
    v = v * (torch.rand((cols, rows), generator=gen, device="cuda") < density)
    if shift or pad:
        ld = rows + pad
        flat = torch.full((shift + ld * cols + 8,), float("nan"), dtype=dtype, device="cuda")
        t = flat.as_strided((cols, rows), (ld, 1), shift)
        t.copy_(v)
    else:
        t = v.to(dtype)
    return t.t() if order == 0 else t


def same(got, want, what):
    assert torch.equal(got.double(), want), f"{what}: {(got.double() - want).abs().max().item()} off"


def run(dtype, order, kn, ci, t, shift=0, pad=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(kn + ci + t)
    F = ints(g, (kn, ci), min(1.0, 30 / ci), dtype, shift, pad, order)
    X = ints(g, (ci, t), 1.0, dtype, shift, pad)
    b = ints(g, (kn, 1), 1.0, dtype)[:, 0]
    R = ints(g, (kn, t), 1.0, dtype, shift, pad)
    dO = ints(g, (kn, t), 0.02, dtype, shift, pad)
    O, Z = lt().linear(F, X, bias=b, activation="relu", residual=R, keep_pre=True)
    f, x, d = F.double(), X.double(), dO.double()
    z = f @ x + b.double()[:, None]
    assert z.abs().max() < 256 and (f.t() @ d).abs().max() < 256     # exact in every type
    same(Z, z, "Z")
    same(O, z.clamp_min(0) + R.double(), "O")
    dX, dF, db = lt().linear_backward(F, X, dO)
    same(dX, f.t() @ d, "dX")
    same(dF, d @ x.t(), "dF")
    same(db, d.sum(1), "dbias")
    dm = d * (z > 0)
    dX, dF, db = lt().linear_backward(F, X, dO, pre=Z, activation="relu")
    same(dX, f.t() @ dm, "dX through relu")
    same(dF, dm @ x.t(), "dF through relu")
    same(db, dm.sum(1), "dbias through relu")


@pytest.mark.parametrize("dtype,order,kernel,kn,ci,t", CASES)
def test_kernels(dtype, order, kernel, kn, ci, t):
    print(f"[kernel] {dtype} order {order} kernel {kernel}: {kn} x {ci}, {t}", flush=True)
    if torch.cuda.get_device_properties(0).multi_processor_count == 256:
        assert lt().linear_choice(dtype, kn, ci, t, order)[5] == kernel
    run(dtype, order, kn, ci, t)


@pytest.mark.parametrize("dtype,order,kernel,kn,ci,t", CASES[::3])
@pytest.mark.parametrize("shift,pad", [(1, 3), (0, 5)])
def test_kernels_unaligned(dtype, order, kernel, kn, ci, t, shift, pad):
    """Odd addresses and leading dimensions: copies, narrow loads, registers."""
    print(f"[kernel unaligned] {dtype} order {order}: {kn} x {ci}, {t} shift {shift} pad {pad}", flush=True)
    run(dtype, order, kn - 1, ci + 1, t, shift, pad)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("order", [0, 1])
@pytest.mark.parametrize("t", [5, 700])
def test_lines_far_apart(dtype, order, t):
    """A leading dimension so large that a tile's offsets pass 32 bits."""
    ld, lines = (1 << 22) + 8, 300
    g = torch.Generator(device="cuda")
    g.manual_seed(7)
    wide = torch.full((ld * lines,), float("nan"), dtype=dtype, device="cuda")
    shape = (lines, 96) if order else (96, lines)
    F = wide.as_strided((lines, 96), (ld, 1))
    F.copy_(ints(g, (lines, 96), 0.2, torch.float32))
    F = F if order else F.t()
    X = ints(g, (shape[1], t), 1.0, dtype)
    same(lt().linear(F, X), F.double() @ X.double(), "O")
    dO = ints(g, (shape[0], t), 0.02, dtype)
    dX, dF, _ = lt().linear_backward(F, X, dO)
    same(dX, F.double().t() @ dO.double(), "dX")
    same(dF, dO.double() @ X.double().t(), "dF")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("t", [2, 700])
def test_long_aligned_lines(dtype, t):
    """Lines far apart but aligned, near the limit of the direct loads on both
    sides: the workspace that is asked for holds what the call takes."""
    g = torch.Generator(device="cuda")
    g.manual_seed(9)
    for ld in ((1 << 20) + 64, (1 << 21) - 64, (1 << 21) + 64):
        F = torch.zeros(ld * 184, dtype=dtype, device="cuda").as_strided((184, 2760), (ld, 1))
        F.copy_(ints(g, (184, 2760), 0.01, torch.float32))
        X, dO = ints(g, (2760, t), 1.0, dtype), ints(g, (184, t), 0.1, dtype)
        same(lt().linear(F, X), F.double() @ X.double(), "O")
        dX, dF, _ = lt().linear_backward(F, X, dO)
        same(dX, F.double().t() @ dO.double(), "dX")
        same(dF, dO.double() @ X.double().t(), "dF")


@pytest.mark.parametrize("order", [0, 1])
@pytest.mark.parametrize("t", [3, 520])
def test_weights_above_four_gib(order, t):
    """65544 x 36000 bfloat16 weights, 4.7 GB: offsets beyond 32 bits."""
    kn, ci = 65544, 36000
    g = torch.Generator(device="cuda")
    g.manual_seed(8)
    F = torch.zeros((kn, ci) if order else (ci, kn), dtype=torch.bfloat16, device="cuda")
    at = torch.randint(0, F.numel(), (2_000_000,), generator=g, device="cuda")
    F.view(-1)[at] = 1.0
    F.view(-1)[-3:] = 1.0                              # the last values of all
    F = F if order else F.t()
    X = ints(g, (ci, t), 1.0, torch.bfloat16)
    O = lt().linear(F, X)
    rows = torch.cat([torch.arange(0, 200), torch.arange(kn // 2, kn // 2 + 100), torch.arange(kn - 200, kn)]).cuda()
    same(O[rows], F[rows].double() @ X.double(), "O")
    del O
    dO = ints(g, (kn, t), 0.02, torch.bfloat16)
    dX, dF, _ = lt().linear_backward(F, X, dO, needs=(True, True, False))
    cols = torch.cat([torch.arange(0, 100), torch.arange(ci - 100, ci)]).cuda()
    same(dX[cols], F[:, cols].double().t() @ dO.double(), "dX")
    same(dF[rows], dO[rows].double() @ X.double().t(), "dF")


def test_gradient_above_two_to_the_31():
    """One tensor of 2.2e9 bfloat16 values; the last of them differs."""
    n = 2_200_000_003
    big = torch.full((n,), 0.5, dtype=torch.bfloat16, device="cuda")
    big[-1] = 3.0
    want = (0.25 * (n - 1) + 9.0) ** 0.5
    norm = lt().clip_grad_norm([big], want / 4)
    assert abs(float(norm) - want) <= 2.0 ** -23 * want
    assert big[0].item() == 0.125 and big[n // 2].item() == 0.125 and big[-1].item() == 0.75 and big[-2].item() == 0.125

"""What the layer operators give their kernels, recorded without a GPU: every
launch stays inside the workspace that was asked for, over sizes on both sides of
every limit up to the largest accepted ones."""
from __future__ import annotations

import os
import random
import re
import shutil

import pytest

import launches
import paper_2005_06410_amd as lt
from paper_2005_06410_amd import build as ltbuild

BF16, F16, F32 = 4, 5, 1
SIZE = {F32: 4, BF16: 2, F16: 2}
W = 1 << 47                                         # the workspace's address
F, X, DO, Z, OUT = (k << 48 for k in (1, 2, 3, 4, 5))
LIMIT = 1 << 24                                     # sizes and leading dimensions lie below it

pytestmark = pytest.mark.skipif(not (os.path.exists("/opt/rocm/bin/hipcc") or shutil.which("hipcc")), reason="hipcc not available")


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(lt.LIB_PATH):
        ltbuild.build()
    return lt.load()


def up(n, step):
    return -(-n // step) * step


def aligned(dtype, lds, shift):
    """Whether the header's aligned = 1 holds."""
    return int(shift == 0 and all(ld * SIZE[dtype] % 16 == 0 and ld * SIZE[dtype] < 1 << 22 for ld in lds))


def forward(lib, dtype, kn, ci, t, order, pad=0, shift=0):
    """(query's bytes, the call with exactly these)."""
    ldf, ldx = (ci if order else kn) + pad, ci + pad
    need = lib.convgemm_linear_workspace(dtype, kn, ci, t, order, aligned(dtype, (ldf, ldx), shift))
    assert need >= 0
    s = shift * SIZE[dtype]
    return need, ("convgemm_linear", (dtype, kn, ci, t, F + s, order, ldf, X + s, ldx, None, 0, None, 0, None, 0, OUT, kn,
                                      W, need, None))


def backward(lib, dtype, kn, ci, t, order, act, pad=0, shift=0, needs=(1, 1, 1)):
    ldf, ldx, ldd = (ci if order else kn) + pad, ci + pad, kn + pad
    need = lib.convgemm_linear_backward_workspace(dtype, kn, ci, t, order, act, aligned(dtype, (ldf, ldx, ldd), shift))
    assert need >= 0
    s = shift * SIZE[dtype]
    dx, df, db = (OUT + (k << 44) if n else None for k, n in enumerate(needs))
    return need, ("convgemm_linear_backward", (dtype, kn, ci, t, F + s, order, ldf, X + s, ldx, DO + s, ldd, Z + s, ldd, act,
                                               dx, ci, df, ci if order else kn, db, W, need, None))


def kind(v):
    return re.match(r"(?:void )?(\w+)", v["kernel"])[1]


def parts_of(v, dtype):
    """The address ranges that a launch writes besides the call's outputs."""
    size, k = SIZE[dtype], kind(v)
    if k == "slope_kernel":
        out = [(v["dZ"], v["lddz"] * v["t"] * size)] if v["lddz"] else []
        return out + ([(v["part"], -(-v["t"] // v["span"]) * v["kn"] * 4)] if v["part"] else [])
    if k == "pad_kernel":
        return [(v[c + "to"], v[c + "lines"] * v[c + "to_ld"] * size) for c in (["a_", "b_"] if v["grid"] > v["a_blocks"] else ["a_"])]
    if k in ("ring_kernel", "wide_kernel") and v["splits"] > 1:
        return [(v["part"], v["splits"] * v["M"] * v["N"] * 4)]
    return []


def check_inside(need, call, code, launched):
    """Every launch writes inside the workspace, and nothing over what a later
    launch of the same product reads."""
    dtype = call[1][0]
    assert code == 0, (call, code)
    dz, copies = [], []
    for v in launched:
        mine = parts_of(v, dtype)
        for at, n in mine:
            assert W <= at and at + n <= W + need, f"{call}: {v['kernel']} writes {at + n - W - need} bytes past the workspace"
        k = kind(v)
        if k == "slope_kernel":
            dz = mine
        if k == "pad_kernel":
            copies = mine
        if k in ("ring_kernel", "wide_kernel"):
            held = dz[:1] + copies + mine
            held = sorted(r for r in held if r[1])
            assert all(a + n <= b for (a, n), (b, _) in zip(held, held[1:])), f"{call}: {v['kernel']} overlaps {held}"
            for operand in (v["A"], v["B"]):
                if operand >= W and operand < F:
                    assert any(operand == a for a, _ in held)
            copies = []


# on both sides of where a line passes what the direct loads reach, and of the limit of the sizes
EDGES = [(1 << 21) - 16, (1 << 21) - 2, 1 << 21, 2200000, (1 << 22) - 8, 1 << 22, 5000001, (1 << 23) - 8, (1 << 23) + 8, LIMIT - 8, LIMIT - 1]


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_backward_stays_inside_for_long_lines(lib, dtype):
    """Many outputs: the library's own dZ has lines as long as they."""
    calls = []
    for long in EDGES:
        for ci, t in [(64, 80), (64, 8), (16, 128), (200, 1), (8, 700)]:
            for order in (0, 1):
                for act in (0, 1, 2):
                    calls.append(backward(lib, dtype, long, ci, t, order, act))
            calls.append(backward(lib, dtype, ci, long, t, 1, 2))
            calls.append(backward(lib, dtype, ci, t, long, 0, 2))
    for (need, call), (code, launched) in zip(calls, launches.record([c for _, c in calls])):
        check_inside(need, call, code, launched)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_everything_stays_inside(lib, dtype):
    """Random sizes, alignments and leading dimensions."""
    rng = random.Random(dtype)
    calls = []
    for _ in range(400):
        kn, ci, t = (int(2 ** rng.uniform(0, 14)) for _ in range(3))
        if rng.random() < 0.4:
            kn, ci = up(kn, 8), up(ci, 8)
        pad, shift = rng.choice([(0, 0), (8, 0), (3, 0), (0, 1), (8, 8), (1 << 20, 0), (1 << 22, 0), (1 << 23, 0)])
        pad = min(pad, LIMIT - 1 - max(kn, ci))
        order = rng.randrange(2)
        calls.append(forward(lib, dtype, kn, ci, t, order, pad, shift))
        calls.append(backward(lib, dtype, kn, ci, t, order, rng.randrange(5), pad, shift))
    for (need, call), (code, launched) in zip(calls, launches.record([c for _, c in calls])):
        check_inside(need, call, code, launched)


def ring_of(name):
    """A direct-loading kernel's operands as (contraction contiguous, lines of a
    stage, values of a line that a stage reaches), and the bytes of a value; None
    where the kernel loads through registers."""
    bits = {"float": 4, "unsigned short": 2, "short": 2}
    if m := re.search(r"wide_kernel<([\w ]+), (\w+), (\w+), \w+>", name):
        size = bits[m[1]]
        return size, [(True, 256, 64) if m[k] == "true" else (False, 64, 256) for k in (2, 3)]
    m = re.search(r"Ring<([\w ]+), (\w+), (\w+), ([\d, ]+)>", name)
    size = bits[m[1]]
    wm, wn, waves_m, waves_n, _, depth, _, width = (int(v) for v in m[4].split(","))
    if width == 0:
        return None
    deep = 128 // size * depth
    return size, [(True, rows, deep) if m[k] == "true" else (False, deep, rows)
                  for k, rows in ((2, 16 * wm * waves_m), (3, 16 * wn * waves_n))]


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_offsets_fit_the_direct_loads(lib, dtype):
    """The 32-bit offsets of a stage, its lanes beyond the operand's end among them,
    lie below the range that says "nowhere"; launches hold fewer than 2^32 threads."""
    rng = random.Random(dtype + 100)
    sizes = [(long, a, b) for long in EDGES for a, b in [(1024, 1024), (512, 512), (64, 80), (8, 8), (200, 1), (3000, 24), (260, 3), (8, 8192), (8192, 1), (1, 4000)]]
    sizes += [(int(2 ** rng.uniform(20, 24)) - 1, int(2 ** rng.uniform(0, 11)), int(2 ** rng.uniform(0, 11))) for _ in range(60)]
    calls = []
    for long, a, b in sizes:
        for kn, ci, t in [(long, a, b), (a, long, b), (a, b, long)]:
            for order in (0, 1):
                for pad in {0, min(1 << 20, LIMIT - 1 - long), min(1 << 23, LIMIT - 1 - long)}:
                    calls.append(forward(lib, dtype, kn, ci, t, order, pad))
                    calls.append(backward(lib, dtype, kn, ci, t, order, 0, pad))
                calls.append(backward(lib, dtype, kn, ci, t, order, 2))
    seen = set()
    for (need, call), (code, launched) in zip(calls, launches.record([c for _, c in calls])):
        check_inside(need, call, code, launched)
        for v in launched:
            assert v["grid"] * v["block"] < 1 << 32, (call, v)
            if kind(v) not in ("ring_kernel", "wide_kernel"):
                continue
            ring = ring_of(v["kernel"])
            seen.add(ring is None)
            if ring is None:
                continue
            size, operands = ring
            for (kc, lines, reach), ld in zip(operands, (v["lda"], v["ldb"])):
                assert ((lines - 1) * ld + reach) * size < 0xfffff000, (call, v)
    assert seen == {True, False}


SUBSETS = [(1, 1, 1), (1, 0, 0), (0, 1, 0), (0, 0, 1), (1, 1, 0), (1, 0, 1), (0, 1, 1), (0, 0, 0)]


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_fewer_outputs_need_no_more(lib, dtype):
    """The bytes that the query names are enough whatever outputs are left out; with
    dbias alone nothing else is written."""
    rng = random.Random(dtype + 200)
    calls = []
    sizes = [(2070, 246, 52), (5361, 186, 7)] + [tuple(int(2 ** rng.uniform(0, 13)) for _ in range(3)) for _ in range(250)]
    for kn, ci, t in sizes:
        order, act, vec = rng.randrange(2), rng.choice([0, 0, 1, 2]), 16 // SIZE[dtype]
        # leading dimensions of whole vectors, extents of any length
        lds = [up(n, vec) for n in (ci if order else kn, ci, kn)]
        for needs in SUBSETS:
            need, (name, args) = backward(lib, dtype, kn, ci, t, order, act, needs=needs)
            args = list(args)
            args[6], args[8], args[10], args[12] = lds[0], lds[1], lds[2], lds[2]
            need = args[-2] = lib.convgemm_linear_backward_workspace(dtype, kn, ci, t, order, act, 1)
            calls.append((needs, need, (name, tuple(args))))
    for (needs, need, call), (code, launched) in zip(calls, launches.record([c for _, _, c in calls])):
        check_inside(need, call, code, launched)
        if needs == (0, 0, 1):
            assert {kind(v) for v in launched} <= {"slope_kernel", "bias_kernel"} and not any(v.get("lddz") for v in launched)
        if needs == (0, 0, 0):
            assert not launched

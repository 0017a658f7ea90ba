"""What the losses give their kernels, recorded without a GPU: every launch stays inside
the workspace that was asked for and reads what an earlier one wrote, over sizes on both
sides of every limit; and the argument checks, which come before any GPU work."""
from __future__ import annotations

import os
import random
import re
import shutil
import subprocess

import pytest

import launches
import paper_2005_06410_amd as lt
from paper_2005_06410_amd import build as ltbuild

BF16, F16, F32 = 4, 5, 1
I32, I64 = 1, 2
SIZE = {F32: 4, BF16: 2, F16: 2}
W = 1 << 47
F, X, B, Y, TOP, LOSS, LSE, G, DX, DF, DB = (k << 48 for k in range(1, 12))
LIMIT = 1 << 24

needs_hipcc = pytest.mark.skipif(not (os.path.exists("/opt/rocm/bin/hipcc") or shutil.which("hipcc")), reason="hipcc not available")


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(lt.LIB_PATH):
        ltbuild.build()
    return lt.load()


@pytest.fixture(scope="module")
def recorder(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("recorder") / "recorder.so")
    subprocess.run([ltbuild.hipcc(), "--offload-arch=gfx950", "--offload-host-only", "-O1", "-fPIC", "-shared", "-std=c++17",
                    "-I" + ltbuild.INCLUDE, "-I" + ltbuild.CSRC, os.path.join(launches.HERE, "loss_recorder.hip"), "-o", out],
                   check=True, capture_output=True, text=True)
    return out


def record(recorder, calls, monkeypatch):
    monkeypatch.setattr(launches, "recorder", lambda: recorder)
    return launches.record(calls)


def up(n, step=256):
    return -(-n // step) * step


def aligned(dtype, lds, shift):
    return int(shift == 0 and all(ld * SIZE[dtype] % 16 == 0 and ld * SIZE[dtype] < 1 << 22 for ld in lds))


def layer(dtype, kn, ci, t, order, pad, shift):
    ldf, ldx, s = max(ci if order else kn, 1) + pad, max(ci, 1) + pad, shift * SIZE[dtype]
    return (dtype, kn, ci, t, F + s, order, ldf, X + s, ldx, B), aligned(dtype, (ldf, ldx), shift)


def teacher(k):
    return (k, TOP, F32, k, Y, I64, k, 2.0) if k else (Y, I64, -100)


def forward(lib, dtype, kn, ci, t, order, k=0, pad=0, shift=0):
    a, al = layer(dtype, kn, ci, t, order, pad, shift)
    need = lib.convgemm_linear_loss_workspace(dtype, kn, ci, t, order, k, al)
    assert need >= 0
    return need, ("convgemm_linear_distill" if k else "convgemm_linear_cross_entropy", a + teacher(k) + (LOSS, LSE, W, need, None))


def backward(lib, dtype, kn, ci, t, order, k=0, pad=0, shift=0, needs=(1, 1, 1)):
    a, al = layer(dtype, kn, ci, t, order, pad, shift)
    need = lib.convgemm_linear_loss_backward_workspace(dtype, kn, ci, t, order, k, al)
    assert need >= 0
    out = [p if n else None for n, p in zip(needs, (DX, DF, DB))]
    return need, ("convgemm_linear_distill_backward" if k else "convgemm_linear_cross_entropy_backward",
                  a + teacher(k) + (LSE, G, 1, out[0], max(ci, 1), out[1], max(ci if order else kn, 1), out[2], W, need, None))


def kind(v):
    return re.match(r"(?:void )?(\w+)", v["kernel"])[1]


def tile_of(v):
    """(rows, columns) of a wave's tile."""
    if "wide_kernel" in v["kernel"]:
        return 128, 64
    m = re.search(r"Ring<[\w ]+, \w+, \w+, (\d+), (\d+),", v["kernel"])
    return 16 * int(m[1]), 16 * int(m[2])


def check_inside(need, call, code, launched):
    """Address ranges that each launch writes in the workspace, against the workspace
    and against what is still read."""
    name, args = call
    dtype, kn, ci, t, _, order = args[:6]
    size, back = SIZE[dtype], "backward" in name
    assert code == 0, (call, code)
    columns = 0
    live = {}                                        # what later launches read: name -> (address, bytes)

    def write(what, at, n, over=()):
        assert W <= at and at + n <= W + need, f"{call}: {what} ends {at + n - W - need} bytes past the workspace"
        for other, (a, m) in live.items():
            if other != what and other not in over and n and m:
                assert at + n <= a or a + m <= at, f"{call}: {what} over {other}"
        live[what] = (at, n)

    def reads(what, at, n=None):
        assert what in live and live[what][0] == at and (n is None or n <= live[what][1]), f"{call}: {what}"

    for v in launched:
        k = kind(v)
        assert v["grid"] * v["block"] < 1 << 32
        if k == "list_kernel":
            bins = -(-kn // 128)
            n = v["grid"]
            assert v["bins"] == bins and v["size"] >= v["k"] and v["size"] <= 1024 and (n == t or not back)
            write("sorted", v["sorted"], n * v["k"] * 4), write("weight", v["weight"], n * v["k"] * 4)
            write("bin", v["bin"], n * (bins + 1) * 2), write("counts", v["counts"], n * 4)
        elif k == "column_kernel":
            write("w", v["w"], t * 4)
            if dtype != F32:
                write("back", v["back"], 4)
        elif k == "input_kernel":
            reads("w", v["w"])
            assert v["ldto"] >= ci and v["t"] == t
            write("x", v["to"], v["ldto"] * t * size)
        elif k == "pad_kernel":
            for c in ["a_", "b_"] if v["grid"] > v["a_blocks"] else ["a_"]:
                fr = v[c + "from"]
                what = "f" if F <= fr < X else "x2" if X <= fr < B else "copy" + c
                write(what, v[c + "to"], v[c + "lines"] * v[c + "to_ld"] * size, over=("copya_", "copyb_"))
        elif k in ("loss_ring_kernel", "loss_wide_kernel"):
            rows, cols = tile_of(v)
            assert v["splits"] == 1 and v["part"] == 0 and v["row0"] % 256 == 0 and v["row0"] + v["M"] <= kn
            n = v["N"]
            assert n == t if back else n <= t
            columns += 0 if back else n
            for operand in (v["A"], v["B"]):
                assert operand >= F or operand == 0 or any(a == operand for a, _ in live.values()) or ci == 0
            if v["k"]:
                reads("sorted", v["index"]), reads("weight", v["weight"]), reads("bin", v["bin"]), reads("counts", v["counts"])
            if back:
                reads("w", v["w"])
                assert v["lse"] == LSE and v["lddz"] >= v["M"] and v["lddz"] * size % 16 == 0
                live.pop("dbpart", None)
                write("dz", v["dZ"], v["lddz"] * t * size)
                if v["db"]:
                    write("dbpart", v["db"], -(-t // cols) * v["M"] * 4)
            else:
                write("sums", v["sums"], -(-v["M"] // rows) * n * 8), write("at", v["at"], n * max(v["k"], 1) * 4)
        elif k in ("shared_loss_kernel", "shared_dz_kernel"):
            reads("part", v["shares"], v["splits"] * v["M"] * v["N"] * 4)
            assert v["N"] == t and v["row0"] + v["M"] <= kn
            columns += 0 if back else t
            if back:
                reads("w", v["w"])
                assert v["lddz"] >= v["M"] and v["lddz"] * size % 16 == 0
                live.pop("dbpart", None)
                write("dz", v["dZ"], v["lddz"] * t * size)
                if v["db"]:
                    write("dbpart", v["db"], -(-t // 8) * v["M"] * 4)
            live.pop("part")
        elif k == "join_loss_kernel":
            if kn:
                reads("sums", v["sums"], v["parts"] * v["N"] * 8), reads("at", v["at"])
                assert live["sums"][1] == v["parts"] * v["N"] * 8
            live.clear()                              # the next round of columns starts over
        elif k == "row_sum_kernel":
            if t:
                reads("dbpart", v["part"], v["parts"] * v["M"] * 4)
                assert live["dbpart"][1] == v["parts"] * v["M"] * 4
        elif k in ("ring_kernel", "wide_kernel"):
            for operand, n in ((v["A"], v["lda"]), (v["B"], v["ldb"])):
                if W <= operand < F and v["K"]:
                    assert any(a == operand for a, _ in live.values())
            if v["part"]:
                write("dxsum" if v["C"] >= DX and v["C"] < DF and (v["adds"] or "dxsum" in live or needs_pieces(launched)) else "part",
                      v["part"], v["splits"] * v["M"] * v["N"] * 4, over=("copya_", "copyb_"))
            if v["C"]:
                live.pop("copya_", None), live.pop("copyb_", None), live.pop("part", None)
        else:
            assert k == "join_kernel", v
    assert back or columns == t or kn == 0
    if back and args[-8] is not None and kn * ci * t:      # dX: every class contributes once
        done = [v for v in launched if kind(v) in ("ring_kernel", "wide_kernel") and DX <= v["C"] < DF]
        assert sum(v["K"] for v in done) == kn
        assert [v["adds"] for v in done] == [0] + [1] * (len(done) - 1)


def needs_pieces(launched):
    return sum(kind(v) in ("loss_ring_kernel", "loss_wide_kernel") for v in launched) > 1


EDGES = [(1 << 20) - 8, 1 << 20, (1 << 20) + 264, (1 << 21) - 2, 2200000, 1 << 22, 5000001, (1 << 23) + 8, LIMIT - 1]


@needs_hipcc
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_everything_stays_inside(lib, recorder, dtype, monkeypatch):
    rng = random.Random(dtype)
    calls = []
    for _ in range(300):
        kn, ci, t = int(2 ** rng.uniform(0, 17)), int(2 ** rng.uniform(0, 13)), int(2 ** rng.uniform(0, 14))
        if rng.random() < 0.4:
            kn, ci = up(kn, 8), up(ci, 8)
        pad, shift = rng.choice([(0, 0), (8, 0), (3, 0), (0, 1), (8, 8), (1 << 20, 0), (1 << 22, 0), (1 << 23, 0)])
        order, k = rng.randrange(2), rng.choice([0, 0, 1, 3, 64, 1000, 1024])
        needs = rng.choice([(1, 1, 1), (1, 1, 1), (1, 0, 0), (0, 1, 0), (0, 0, 1), (1, 1, 0), (0, 1, 1), (1, 0, 1)])
        calls.append(forward(lib, dtype, kn, ci, t, order, k, pad, shift))
        calls.append(backward(lib, dtype, kn, ci, t, order, k, pad, shift, needs))
    for (need, call), (code, launched) in zip(calls, record(recorder, [c for _, c in calls], monkeypatch)):
        check_inside(need, call, code, launched)


@needs_hipcc
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_long_lines_and_empty_extents_stay_inside(lib, recorder, dtype, monkeypatch):
    calls = []
    sizes = [(a, b, c) for long in EDGES for a, b, c in [(long, 64, 80), (long, 16, 3), (16, long, 5), (1000, long, 80), (200, 24, long)]]
    # more logits than one round holds
    sizes += [(1 << 18, 16, 1 << 21), (131073, 24, (1 << 20) + 7), (LIMIT - 1, 8, 65535), (3, 5, LIMIT - 1)]
    sizes += [(0, 5, 5), (5, 0, 5), (5, 5, 0), (0, 0, 3), (1, 1, 1)]
    for kn, ci, t in sizes:
        for order in (0, 1):
            for k in (0, 2):
                for pad in (0, 1):
                    pad = min(pad, LIMIT - 1 - max(kn, ci))
                    calls.append(forward(lib, dtype, kn, ci, t, order, k, pad))
                    calls.append(backward(lib, dtype, kn, ci, t, order, k, pad))
    for (need, call), (code, launched) in zip(calls, record(recorder, [c for _, c in calls], monkeypatch)):
        check_inside(need, call, code, launched)


@needs_hipcc
def test_every_kernel_is_reached(lib, recorder, monkeypatch):
    """Both ends exist for the tiles and loads that the layer's own products have with a
    contiguous contraction on the right, and sizes reach all of them."""
    rng = random.Random(7)
    seen = {}
    for dtype in (F32, BF16, F16):
        calls = []
        for order in (0, 1):
            for _ in range(700):
                kn, ci, t = int(2 ** rng.uniform(0, 17)), int(2 ** rng.uniform(0, 13)), int(2 ** rng.uniform(0, 14))
                if rng.random() < 0.75:
                    kn, ci = up(kn, 8), up(ci, 8)
                calls += [forward(lib, dtype, kn, ci, t, order)[1], backward(lib, dtype, kn, ci, t, order)[1]]
            for t in (5, 20, 80):
                calls += [forward(lib, dtype, 24, (1 << 23) + 16, t, order)[1], backward(lib, dtype, 24, (1 << 23) + 16, t, order)[1]]
        for code, launched in record(recorder, calls, monkeypatch):
            assert code == 0
            for v in launched:
                if kind(v).startswith("loss_"):
                    seen.setdefault(v["kernel"].replace("linear::", ""), v)
    rings = {re.search(r"(\w+End), .*Ring<([\w ]+), (\w+), \w+, ([\d, ]+)>", k).groups() for k in seen if "ring" in k}
    for end in ("StatsEnd", "SlopeEnd"):
        for kind_ in ("float", "short", "unsigned short"):
            for kc in ("true", "false"):
                mine = {r[3] for r in rings if r[:3] == (end, kind_, kc)}
                # eight tiles for any type, one for a contiguous contraction, two for fp32, three through registers
                want = 8 + (kc == "true") + 2 * (kind_ == "float") + 3
                assert len(mine) >= want, (end, kind_, kc, sorted(mine))
    assert sum("loss_wide_kernel" in k for k in seen) == 8


GOOD = dict(dtype=F32, kn=4, ci=3, t=2, F=16, order=0, ldf=4, X=16, ldx=3, bias=None)
LABELS = dict(labels=16, itype=I64, ignore=-100)
TEACHER = dict(k=2, top=16, ttype=BF16, ldtop=2, index=16, itype=I32, ldi=2, temperature=1.0)
FORWARD = dict(loss=16, lse=16, ws=16, bytes=1 << 40, stream=None)
GRADS = dict(lse=16, g=16, ginc=1, dX=16, lddx=3, dF=16, lddf=4, db=16, ws=16, bytes=1 << 40, stream=None)
LAYER_FAULTS = [({"dtype": 0}, -1), ({"kn": -1}, -2), ({"kn": LIMIT}, -2), ({"ci": -1}, -3), ({"t": -1}, -4), ({"t": LIMIT}, -4), ({"F": None}, -5),
                ({"order": 2}, -6), ({"ldf": 3}, -7), ({"X": None}, -8), ({"ldx": 2}, -9)]
LABEL_FAULTS = [({"labels": None}, -11), ({"itype": 3}, -12)]
TEACHER_FAULTS = [({"k": 0}, -11), ({"k": 1025}, -11), ({"top": None}, -12), ({"ttype": 2}, -13), ({"ldtop": 1}, -14), ({"index": None}, -15), ({"itype": 0}, -16),
                  ({"ldi": 1}, -17), ({"temperature": 0.0}, -18), ({"temperature": float("nan")}, -18), ({"temperature": 1e300}, -18), ({"temperature": 1e-45}, -18), ({"temperature": 1e-30}, -18)]


def faults(first):
    return [({"lse": None}, -first), ({"g": None}, -first - 1), ({"ginc": 2}, -first - 2), ({"lddx": 2}, -first - 4), ({"lddf": 3}, -first - 6),
            ({"ws": None}, -first - 8), ({"ws": 8}, -first - 8), ({"bytes": 16}, -first - 9)]


@pytest.mark.parametrize("name,args,list_", [
    ("convgemm_linear_cross_entropy", {**GOOD, **LABELS, **FORWARD},
     LAYER_FAULTS + LABEL_FAULTS + [({"loss": None}, -14), ({"lse": None}, -15), ({"ws": None}, -16), ({"ws": 24}, -16), ({"bytes": 8}, -17)]),
    ("convgemm_linear_distill", {**GOOD, **TEACHER, **FORWARD},
     LAYER_FAULTS + TEACHER_FAULTS + [({"loss": None}, -19), ({"lse": None}, -20), ({"ws": None}, -21), ({"bytes": 8}, -22)]),
    ("convgemm_linear_cross_entropy_backward", {**GOOD, **LABELS, **GRADS}, LAYER_FAULTS + LABEL_FAULTS + faults(14)),
    ("convgemm_linear_distill_backward", {**GOOD, **TEACHER, **GRADS}, LAYER_FAULTS + TEACHER_FAULTS + faults(19)),
])
def test_argument_checks(lib, name, args, list_):
    for change, code in list_:
        assert getattr(lib, name)(*dict(args, **change).values()) == code, change


def test_workspace_queries(lib):
    for fn in (lib.convgemm_linear_loss_workspace, lib.convgemm_linear_loss_backward_workspace):
        assert fn(9, 4, 4, 4, 0, 0, 1) == -1 and fn(F32, 4, 4, 4, 2, 0, 1) == -5 and fn(F32, 4, 4, 4, 0, 1025, 1) == -6
        for kn, ci, t in [(1000, 4096, 80), (32000, 1001, 5), (10007, 64, 777), (50, 70001, 3)]:
            for order in (0, 1):
                for k in (0, 17):
                    assert fn(BF16, kn, ci, t, order, k, 0) >= fn(BF16, kn, ci, t, order, k, 1) > 0
    # the logits are not kept: 131072 classes by 8192 tokens would be 2 GB in bf16
    assert lt.load().convgemm_linear_loss_workspace(BF16, 131072, 4096, 8192, 1, 0, 1) < 80 << 20
    assert lt.load().convgemm_linear_loss_backward_workspace(BF16, 131072, 4096, 8192, 1, 0, 1) < 512 << 20

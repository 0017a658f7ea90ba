"""The lists that the norm and the clipping give their kernels, recorded without a
GPU: counts of chunks at the limits of what is accepted."""
from __future__ import annotations

import os
import shutil

import pytest

import launches
import paper_2005_06410_amd as lt
from paper_2005_06410_amd import build as ltbuild

BF16, F32 = 4, 1
MOST = (1 << 37) - 1                                # values of the largest tensor that is accepted

pytestmark = pytest.mark.skipif(not (os.path.exists("/opt/rocm/bin/hipcc") or shutil.which("hipcc")), reason="hipcc not available")


@pytest.mark.parametrize("sizes", [[1, 0, 4097], [MOST], [MOST] * 240, [MOST] * 500, [5] * 239 + [MOST], [1 << 30] * 200 + [3] * 100])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_chunks(sizes, dtype):
    if not os.path.exists(lt.LIB_PATH):
        ltbuild.build()
    n = len(sizes)
    need = lt.load().convgemm_grad_workspace(n)
    g, out = {"of": "p", "values": [1 << 40] * n}, {"of": "p", "values": [1 << 41] * n}
    sz, dt = {"of": "q", "values": sizes}, {"of": "i", "values": [dtype] * n}
    (c1, norm), (c2, clip) = launches.record([("convgemm_grad_norm", (n, g, sz, dt, 16, 1 << 42, need, None)),
                                              ("convgemm_grad_clip", (n, g, out, sz, dt, 1.0, 16, 1 << 42, need, None))])
    assert c1 == c2 == 0
    size = 4 if dtype == F32 else 2
    for launched, name in ((norm, "norm_kernel"), (clip, "norm_kernel"), (clip, "scale_kernel")):
        mine = [v for v in launched if name in v["kernel"]]
        left = [s for s in sizes if s]
        assert len(mine) * 2048 * 8 <= need         # one partial sum for each workgroup
        for v in mine:
            want = [-(-s * size // v["chunk"]) for s in left[:v["count"]]]
            assert v["chunks"] == want and v["last"] == sum(want)
            assert v["grid"] == min(v["last"], 2048) and v["last"] < 1 << 31
            left = left[v["count"]:]
        assert not left

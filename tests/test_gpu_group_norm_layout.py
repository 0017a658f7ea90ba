"""Group norm's C calls: what they write and nothing else, and results in the place of an
input."""
from __future__ import annotations

import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = {torch.float32: 1, torch.bfloat16: 4, torch.float16: 5}
SILU = 4
# (c, s, b), groups: features in a wave and in a workgroup; in a workgroup's registers; in chunks, and
# with their channels joined first; whole and ragged channels of each
LAYOUTS = [((1000, 1, 41), 8), ((1001, 1, 9), 7), ((8192, 1, 3), 1), ((9001, 1, 5), 1), ((96, 42, 5), 8), ((90, 45, 7), 9), ((3, 35, 20), 3),
           ((30, 22650, 2), 5), ((37, 22650, 2), 1), ((2000, 1600, 1), 1), ((515, 4900, 2), 1)]


def lt():
    import paper_2005_06410_amd as m
    return m


class Map:
    """A (c, s, b) map with `pad` values behind each position and `gap` behind each image."""

    def __init__(self, shape, dtype, pad, gap, fill=9.0, values=None):
        c, s, b = shape
        self.ld, self.ldb = c + pad, s * (c + pad) + gap
        self.flat = torch.full((b * self.ldb + 8,), fill, dtype=dtype, device="cuda")
        self.map = self.flat.as_strided(shape, (1, self.ld, self.ldb))
        if values is not None:
            self.map.copy_(values)
        self.args = (self.flat.data_ptr(), self.ld, self.ldb)

    def rest(self):
        """What lies outside the map's values."""
        held = torch.zeros_like(self.flat, dtype=torch.bool)
        held.as_strided(self.map.shape, self.map.stride()).fill_(True)
        return self.flat[~held]


class Call:
    """Inputs of both calls, and the calls with exactly the bytes that the queries name, in
    a buffer whose other bytes have to stay."""

    def __init__(self, shape, groups, dtype):
        c, s, b = shape
        g = torch.Generator(device="cuda").manual_seed(c + s)
        self.x, self.dO = (torch.randn(shape, generator=g, device="cuda").to(dtype) for _ in range(2))
        self.w, self.bias = ((at + 0.3 * torch.randn(c, generator=g, device="cuda")).to(dtype) for at in (1, 0))
        self.shape, self.dtype, self.size = shape, dtype, (TYPES[dtype], c, s, b, groups)
        self.mean, self.rstd = (torch.zeros((b, groups), device="cuda") for _ in range(2))

    def launch(self, name, *args):
        lib = lt().load()
        need = getattr(lib, name + "_workspace")(*self.size)
        buffer = torch.full((need + 512,), 77, dtype=torch.uint8, device="cuda")
        code = getattr(lib, name)(*self.size, *args, buffer.data_ptr() + 256 if need else 0, need, torch.cuda.current_stream().cuda_stream)
        assert code == 0
        assert (buffer[:256] == 77).all() and (buffer[256 + need:] == 77).all()

    def forward(self, x, o):
        self.launch("convgemm_group_norm", *x.args, self.w.data_ptr(), self.bias.data_ptr(), 1e-5, SILU, *o.args, self.mean.data_ptr(),
                    self.rstd.data_ptr())

    def backward(self, x, dO, dI):
        dw, db = torch.zeros_like(self.w), torch.zeros_like(self.w)
        self.launch("convgemm_group_norm_backward", *x.args, *dO.args, self.w.data_ptr(), self.bias.data_ptr(), SILU, self.mean.data_ptr(),
                    self.rstd.data_ptr(), *dI.args, dw.data_ptr(), db.data_ptr())
        return dw, db


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("shape,groups", LAYOUTS)
def test_only_the_maps_are_written(shape, groups, dtype):
    """Maps with room between positions and images: what lies there stays, and the results are
    those of maps without."""
    call = Call(shape, groups, dtype)
    results = []
    for pad, gap in [(0, 0), (3, 5), (8, 16), (0, 7)]:
        x, dO = Map(shape, dtype, pad, gap, torch.nan, call.x), Map(shape, dtype, gap, pad, torch.nan, call.dO)
        o, dI = Map(shape, dtype, pad, gap), Map(shape, dtype, gap, pad)
        call.forward(x, o)
        dw, db = call.backward(x, dO, dI)
        assert (o.rest() == 9).all() and (dI.rest() == 9).all()
        assert torch.equal(x.map, call.x) and torch.equal(dO.map, call.dO)
        results.append((o.map, call.mean.clone(), call.rstd.clone(), dI.map, dw, db))
    for other in results[1:]:
        for a, v in zip(other, results[0]):
            assert torch.equal(a, v)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("shape,groups", LAYOUTS)
def test_gradients_in_the_place_of_an_input(shape, groups, dtype):
    """dI may be dO or I itself."""
    call = Call(shape, groups, dtype)
    for pad, gap in [(0, 0), (3, 5)]:
        x, dO = Map(shape, dtype, pad, gap, values=call.x), Map(shape, dtype, pad, gap, values=call.dO)
        o, dI = Map(shape, dtype, pad, gap), Map(shape, dtype, pad, gap)
        call.forward(x, o)
        want = call.backward(x, dO, dI)
        for place in (0, 1):
            inputs = [Map(shape, dtype, pad, gap, values=v) for v in (call.x, call.dO)]
            got = call.backward(*inputs, inputs[place])
            assert torch.equal(inputs[place].map, dI.map) and torch.equal(inputs[1 - place].map, (call.x, call.dO)[1 - place])
            assert (inputs[place].rest() == 9).all()
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        call.forward(x, x)
        assert torch.equal(x.map, o.map) and (x.rest() == 9).all()

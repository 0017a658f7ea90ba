"""Whether two maps share a value, against the sets of their addresses; and group norm
between the channels of one buffer."""
from __future__ import annotations

import random

import pytest
import torch

import paper_2005_06410_amd as lt


def test_maps_that_meet():
    r = random.Random(2)
    seen = {True: 0, False: 0}
    undecided = 0
    for _ in range(60000):
        c, s, b = r.randrange(1, 4), r.randrange(1, 5), r.randrange(1, 4)
        ldx = c + r.randrange(3) * r.randrange(4)
        ldbx = (s - 1) * ldx + c + r.randrange(3) * r.randrange(8)
        ldo, ldbo = ldx, ldbx
        if r.random() < 0.4:
            ldo = c + r.randrange(3) * r.randrange(4)
            ldbo = (s - 1) * ldo + c + r.randrange(3) * r.randrange(8)
        if r.random() < 0.3:                                    # one run of positions
            ldbx, ldbo = s * ldx, s * ldo
        x, o = r.randrange(40), r.randrange(40)
        sets = [{at + n * ldb + p * ld + k for n in range(b) for p in range(s) for k in range(c)} for at, ld, ldb in
                ((x, ldx, ldbx), (o, ldo, ldbo))]
        want = bool(sets[0] & sets[1])
        got = lt._maps_meet(c, s, b, x, ldx, ldbx, o, ldo, ldbo)
        if got and not want:                                    # only where both have gaps and lie apart differently
            undecided += 1
            assert (ldx, ldbx) != (ldo, ldbo)
        else:
            assert got == want, (c, s, b, x, ldx, ldbx, o, ldo, ldbo)
        seen[want] += 1
    assert min(seen.values()) > 10000 and undecided < 6000
    assert not lt._maps_meet(0, 3, 2, 5, 4, 12, 5, 4, 12)


@pytest.mark.gpu
@pytest.mark.parametrize("c,groups", [(24, 6), (23, 1), (3, 3)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_into_other_channels_of_the_same_buffer(dtype, c, groups):
    """The first c channels of a buffer, normed into the c behind them at the same positions."""
    g = torch.Generator(device="cuda").manual_seed(1)
    for h, w, b in [(5, 6, 3), (150, 151, 2), (1, 1, 70), (5, 6, 1)]:
        whole = torch.randn((b, w, h, 2 * c + 2), generator=g, device="cuda").to(dtype).permute(3, 2, 1, 0)
        before = whole.clone(memory_format=torch.preserve_format)
        x, out = whole[:c], whole[c:2 * c]
        want, mean, rstd = lt.group_norm(before[:c], groups, activation="relu")
        got = lt.group_norm(x, groups, activation="relu", out=out)
        assert got[0] is out and torch.equal(out, want) and torch.equal(got[1], mean) and torch.equal(got[2], rstd)
        assert torch.equal(whole[:c], before[:c]) and torch.equal(whole[2 * c:], before[2 * c:])
        for first in (1, c - 1):                                # some channels in common
            with pytest.raises(ValueError):
                lt.group_norm(x, groups, out=whole[first:first + c])
        if h > 1:                                               # the next position of the same channels
            strides = (1, whole.stride(1), whole.stride(3))
            flat, moved = (whole.as_strided((c, h * w - 1, b), strides, whole.storage_offset() + at) for at in (0, strides[1]))
            with pytest.raises(ValueError):
                lt.group_norm(flat, groups, out=moved)

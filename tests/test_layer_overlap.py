"""Whether two sets of lines share a value, against the sets themselves."""
from __future__ import annotations

import random

import paper_2005_06410_amd as lt


def test_lines_that_meet():
    r = random.Random(1)
    seen = {True: 0, False: 0}
    for _ in range(20000):
        a, b = r.randrange(12), r.randrange(12)
        alen, blen, alines, blines = (r.randrange(5) for _ in range(4))
        ald = max(alen, 1) + r.randrange(4)
        bld = max(ald, blen, 1) if r.random() < 0.6 else max(blen, 1) + r.randrange(4)
        want = bool({a + i + j * ald for i in range(alen) for j in range(alines)}
                    & {b + i + j * bld for i in range(blen) for j in range(blines)})
        got = lt._meet(a, alen, alines, ald, b, blen, blines, bld)
        undecided = alines > 1 and blines > 1 and ald != alen and bld != blen and ald != bld
        assert got == want or (undecided and not got), (a, alen, alines, ald, b, blen, blines, bld)
        seen[got] += 1
    assert min(seen.values()) > 1000

"""The tests of the 8-bit product against its plan (no GPU): sizes that are there to run a kernel run it, and no kernel that
the plan takes somewhere in the range of sizes is without one."""
import random

import pytest

import linear_plan as lp
from paper_2007_06919_amd import aqd

TYPES = (aqd.F32, aqd.F16, aqd.BF16)


@pytest.mark.parametrize("kernel, act, split, past, rows, n, k, ld", lp.COVER)
def test_a_size_reaches_its_kernel(kernel, act, split, past, rows, n, k, ld):
    for t in TYPES:
        shape, parts, _ = lp.plan(lp.args(rows, n, k, t, act, ld, ld), aqd.QLIN_WORKSPACE_BYTES if split else 0)
        assert (lp.NAMES[shape], parts > 1) == (lp.NAMES[kernel], split)
        assert lp.stored_past(shape, parts, rows, n, t) == past


def test_every_kernel_that_the_plan_takes_has_a_size():
    rng = random.Random(1)

    def size(low, high):
        v = low * (high / low) ** rng.random()
        step = 1 if v < 32 else rng.choice([1, 16, 64])
        return max(low, min(high, round(v / step) * step))

    form = lambda shape, act, split, past, words: (lp.NAMES[shape], act, split, past, words if shape == lp.FEW16 else None)
    covered = {form(kernel, act, split, past, ld % 4 == 0) for kernel, act, split, past, _, _, _, ld in lp.COVER}
    for _ in range(100000):
        rows, n, k = size(1, 20000), size(1, 20000), size(1, 131071 if rng.random() < 0.15 else 20000)
        act, t, words = rng.randrange(2), rng.choice(TYPES), rng.random() < 0.5
        ld = -(-k // 4) * 4 if words else k | 1
        for room in (0, aqd.QLIN_WORKSPACE_BYTES):
            shape, parts, _ = lp.plan(lp.args(rows, n, k, t, act, ld, ld), room)
            found = form(shape, act, parts > 1, lp.stored_past(shape, parts, rows, n, t), words)
            assert found in covered, (found, rows, n, k, ld, t, room)


def test_a_plan_stays_within_its_workspace():
    rng, less = random.Random(2), 0
    for _ in range(20000):
        rows, n, k = (int(high ** rng.random()) for high in (4000, 8000, 131071))
        act, t = rng.randrange(2), rng.choice(TYPES)
        full = aqd.qlin_workspace(rows, n, k, t, act)
        for room in (0, 16, full // 4, full // 2, max(0, full - 16), full):
            shape, parts, size = lp.plan(lp.args(rows, n, k, t, act), room)
            assert size <= room and (size > 0) == (parts > 1)
            # the sums of each part, [rows][halves][n up to 4], as the kernels lay them out
            assert parts == 1 or size == 4 * parts * rows * (2 if act else 1) * (-(-n // 4) * 4)
            less += 0 < size < full
    assert less   # less room than asked for may still split

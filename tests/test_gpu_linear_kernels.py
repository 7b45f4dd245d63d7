"""Every kernel of the 8-bit product, split and whole, with every type of y, against 64 bits: the sizes that reach them
(linear_plan.COVER; test_linear_plan.py holds them to the plan), rows of codes that end in junk, nothing written outside of y and
the workspace. Tolerances as in test_gpu_linear.py."""
import math

import pytest

import linear_plan as lp
from paper_2007_06919_amd import aqd

pytestmark = pytest.mark.gpu

TYPES = {"f32": (aqd.F32, 2.0 ** -24, 2.0 ** -150), "f16": (aqd.F16, 2.0 ** -11, 2.0 ** -25), "bf16": (aqd.BF16, 2.0 ** -8, 2.0 ** -134)}
GUARD = 256   # elements around an output


class Product:
    def __init__(self, torch, rows, n, k, ld, t, act, bias, whole=False):
        g = torch.Generator(device="cuda").manual_seed(rows * 31 + n * 17 + k + act)
        self.rows, self.n, self.k, self.act, self.ld = rows, n, k, act, ld
        self.type, self.half, self.least = TYPES[t]
        wide = 2 * n if act else n
        self.x, self.w = (torch.randint(-128, 128, (r, ld), generator=g, device="cuda", dtype=torch.int8) for r in (rows, wide))
        self.sx = (torch.rand(rows, generator=g, device="cuda") + 0.5) / 74
        self.sw = (torch.rand(wide, generator=g, device="cuda") + 0.5) / (74 * math.sqrt(k))
        self.bias = torch.randn(wide, generator=g, device="cuda") if bias else None
        self.dtype = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[t]
        self.ld_y = n if whole else n + 3
        self.first = GUARD if whole else GUARD + 1   # 256 elements: whole lines in each type

    def args(self):
        return lp.args(self.rows, self.n, self.k, self.type, self.act, self.ld, self.ld, self.ld_y, self.x.data_ptr(), self.w.data_ptr())

    def run(self, torch, room):
        """y for a workspace of `room` bytes, with junk around both."""
        buf = torch.full((self.first + self.rows * self.ld_y + GUARD,), 5, dtype=self.dtype, device="cuda")
        work = torch.full((room + GUARD,), 0x55, dtype=torch.uint8, device="cuda")
        y = buf[self.first:self.first + self.rows * self.ld_y].view(self.rows, self.ld_y)[:, :self.n]
        aqd.qlin_run(self.rows, self.n, self.k, self.type, self.act, self.x, self.ld, self.sx, self.w, self.ld, self.sw, self.bias, y,
                     self.ld_y, work if room else None, room)
        out = y.clone()
        y.fill_(5)
        assert bool((buf == 5).all()) and bool((work[room:] == 0x55).all())
        return out

    def check(self, torch, y):
        w = self.w[:, :self.k].double().t().contiguous()
        step = max(1, (1 << 27) // max(w.shape[1], self.k))
        for at in range(0, self.rows, step):
            x, sx = self.x[at:at + step, :self.k].double(), self.sx[at:at + step].double()
            p = torch.mm(x, w) * sx[:, None] * self.sw.double()   # the sums are exact: integers below 2^53
            z = p if self.bias is None else p + self.bias.double()
            ez = (4 * p.abs() + z.abs()) * 2.0 ** -24
            want, tol = z, ez
            if self.act:
                gate, v, eg, ev = z[:, :self.n], z[:, self.n:], ez[:, :self.n], ez[:, self.n:]
                silu = gate / (1 + torch.exp(-gate))
                want = silu * v
                tol = v.abs() * (1.1 * eg + silu.abs() * (gate.abs() + 4) * 2.0 ** -22) + silu.abs() * ev + want.abs() * 2.0 ** -23
            tol = tol * 1.01 + want.abs() * self.half * 1.01 + self.least
            off = (y[at:at + step].double() - want).abs() - tol
            assert bool((off <= 0).all()), f"{int((off > 0).sum())} of {off.numel()} off in rows {at} on"


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("kernel, act, split, past, rows, n, k, ld", lp.COVER)
def test_kernel(kernel, act, split, past, rows, n, k, ld, t):
    import torch
    case = Product(torch, rows, n, k, ld, t, act, bias=(rows + n + k + len(t)) % 2 == 0, whole=past)
    room = aqd.qlin_workspace(rows, n, k, case.type, act, ld, ld, case.ld_y) if split else 0
    shape, parts, _ = lp.plan(case.args(), room)
    assert (lp.NAMES[shape], parts > 1) == (lp.NAMES[kernel], split)
    y = case.run(torch, room)
    case.check(torch, y)
    if split:
        assert torch.equal(y, case.run(torch, 0)), "the split sum differs from the whole one"


@pytest.mark.parametrize("act, rows, n, k, ld", [(0, 192, 1023, 16384, 16384), (1, 192, 1023, 16384, 16384), (0, 300, 500, 5003, 5004),
                                                 (1, 70, 333, 9000, 9000), (1, 23, 65, 20001, 20001), (0, 192, 1023, 16383, 16383),
                                                 (1, 300, 1023, 9001, 9001)])
def test_less_workspace_than_asked_for(act, rows, n, k, ld):
    """The same bits for any workspace, and nothing written past it: with less room the sum is split less, or not at all."""
    import torch
    case = Product(torch, rows, n, k, ld, "bf16", act, bias=True)
    full = aqd.qlin_workspace(rows, n, k, case.type, act, ld, ld, case.ld_y)
    rooms = [full, full - 16, full // 2 // 16 * 16, full // 4 // 16 * 16, 16, 0]
    plans = [lp.plan(case.args(), room) for room in rooms]
    assert plans[0][1] > 1 and any(1 < p[1] and p[2] < full for p in plans[1:])
    whole = case.run(torch, 0)
    case.check(torch, whole)
    for room in rooms:
        assert torch.equal(case.run(torch, room), whole), room

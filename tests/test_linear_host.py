"""Refusals of the 8-bit linear layers' entry points: they come from the host before any
launch, so none of this needs a GPU. Addresses here are never followed."""
import ctypes

import pytest

import linear_plan
from paper_2007_06919_amd import aqd

A = 1 << 20   # an address for each tensor, far from the others
ADDR = {name: A * (i + 1) for i, name in enumerate(("x", "residual", "weight", "sum", "codes", "scales", "x_scales",
                                                    "w", "w_scales", "bias", "y", "workspace"))}


def rows_call(**kw):
    d = dict(rows=4, cols=32, type=aqd.F32, ld_x=0, ld_codes=0, **ADDR)
    d.update(kw)
    aqd.qrows_run(d["rows"], d["cols"], d["type"], d["x"], d["ld_x"], d["codes"], d["ld_codes"], d["scales"], 0)


def norm_call(**kw):
    d = dict(rows=4, cols=32, type=aqd.BF16, eps=1e-5, ld_x=0, ld_residual=0, ld_sum=0, ld_codes=0, **ADDR)
    d.update(kw)
    aqd.qnorm_run(d["rows"], d["cols"], d["type"], d["eps"], d["x"], d["ld_x"], d["residual"], d["ld_residual"],
                  d["weight"], d["sum"], d["ld_sum"], d["codes"], d["ld_codes"], d["scales"], 0)


def lin_call(**kw):
    d = dict(rows=4, n=8, k=32, type=aqd.F16, act=aqd.QLIN_PLAIN, ld_x=0, ld_w=0, ld_y=0, ws_bytes=0, **ADDR)
    d.update(kw)
    aqd.qlin_run(d["rows"], d["n"], d["k"], d["type"], d["act"], d["x"], d["ld_x"], d["x_scales"], d["w"], d["ld_w"],
                 d["w_scales"], d["bias"], d["y"], d["ld_y"], d["workspace"], d["ws_bytes"], 0)


def refused(call, status=aqd.AQD_ERR_INVALID, **kw):
    with pytest.raises(aqd.AqdError) as e:
        call(**kw)
    assert e.value.status == status and aqd.last_error()


@pytest.mark.parametrize("bad", [
    dict(rows=-1), dict(cols=0), dict(type=3), dict(type=-1), dict(ld_x=31), dict(ld_codes=-32), dict(ld_x=1 << 60),
    dict(x=None), dict(codes=None), dict(scales=None), dict(x=A + 2), dict(scales=ADDR["scales"] + 1),
    dict(codes=A + 4 * 32 * 4 - 1), dict(scales=ADDR["codes"] + 4 * 31), dict(scales=A), dict(codes=A),
])
def test_qrows_refuses(bad):
    refused(rows_call, **bad)


@pytest.mark.parametrize("bad", [
    dict(eps=-1e-6), dict(eps=float("nan")), dict(eps=float("inf")), dict(weight=None), dict(ld_residual=8),
    dict(ld_sum=8), dict(residual=ADDR["residual"] + 1), dict(sum=ADDR["sum"] + 1), dict(weight=ADDR["weight"] + 1),
    # sum in place of an input, but not exactly: another stride, a shifted start; over the weight; codes over sum
    dict(sum=ADDR["x"], ld_sum=40), dict(sum=ADDR["residual"] + 2), dict(sum=ADDR["weight"]), dict(codes=ADDR["sum"] + 6),
    dict(scales=ADDR["weight"]), dict(x=None), dict(cols=-1),
])
def test_qnorm_refuses(bad):
    refused(norm_call, **bad)


@pytest.mark.parametrize("bad", [
    dict(rows=-1), dict(n=0), dict(k=0), dict(type=7), dict(act=2), dict(ld_x=31), dict(ld_w=16), dict(ld_y=7),
    dict(x=None), dict(w=None), dict(x_scales=None), dict(w_scales=None), dict(y=None),
    dict(y=ADDR["y"] + 1), dict(x_scales=ADDR["x_scales"] + 2), dict(bias=ADDR["bias"] + 3),
    dict(workspace=ADDR["workspace"] + 8), dict(y=ADDR["x"]), dict(y=ADDR["w"] + 8 * 32 - 2), dict(y=ADDR["bias"]),
    dict(n=1 << 31 - 1, act=aqd.QLIN_SILU_GATE),
])
def test_qlin_refuses(bad):
    refused(lin_call, **bad)


def test_qlin_refuses_sums_that_may_leave_int32():
    refused(lin_call, aqd.AQD_ERR_UNSUPPORTED, k=131072)
    with pytest.raises(aqd.AqdError):
        aqd.qlin_workspace(4, 8, 131072, aqd.F32, aqd.QLIN_PLAIN)


def test_a_null_description_is_refused():
    L = aqd.lib()
    size = ctypes.c_size_t(5)
    assert L.qrows_run(None, A, A, A, None) == aqd.AQD_ERR_INVALID
    assert L.qnorm_run(None, A, A, A, A, A, A, None) == aqd.AQD_ERR_INVALID
    assert L.qlin_run(None, A, A, A, A, A, A, A, 0, None) == aqd.AQD_ERR_INVALID
    assert L.qlin_workspace(None, ctypes.byref(size)) == aqd.AQD_ERR_INVALID
    d = aqd.QlinDesc(4, 8, 32, aqd.F32, aqd.QLIN_PLAIN, 0, 0, 0)
    assert L.qlin_workspace(ctypes.byref(d), None) == aqd.AQD_ERR_INVALID


def test_no_rows_is_no_work():
    rows_call(rows=0, x=None, codes=None, scales=None)
    norm_call(rows=0, x=None)
    lin_call(rows=0, x=None, w=None, y=None)
    assert aqd.qlin_workspace(0, 8, 4096, aqd.F32, aqd.QLIN_PLAIN) == 0


@pytest.mark.parametrize("act", [aqd.QLIN_PLAIN, aqd.QLIN_SILU_GATE])
def test_the_workspace_has_a_bound(act):
    split = 0
    for rows in (1, 3, 16, 17, 64, 65, 128, 200, 512, 1024, 5000, 100000):
        for n in (1, 5, 64, 720, 4096, 16384):
            for k in (1, 64, 515, 4096, 16384, 131071):
                b = aqd.qlin_workspace(rows, n, k, aqd.F32, act)
                assert 0 <= b <= aqd.QLIN_WORKSPACE_BYTES
                split += b > 0
    assert split


def test_real_types():
    import torch
    assert [aqd.real_type(torch.empty(0, dtype=t)) for t in (torch.float32, torch.float16, torch.bfloat16)] == \
        [aqd.F32, aqd.F16, aqd.BF16]
    assert aqd.real_type(torch.float16) == aqd.F16
    with pytest.raises(TypeError):
        aqd.real_type(torch.empty(0, dtype=torch.int8))


@pytest.mark.parametrize("call, bad", [
    (rows_call, dict(ld_x=1 << 62)), (rows_call, dict(ld_codes=1 << 60)), (norm_call, dict(ld_x=1 << 61, ld_sum=1 << 61, sum=A + 8)),
    (norm_call, dict(type=aqd.F32, ld_x=1 << 62, ld_sum=1 << 62, sum=A + 64)), (lin_call, dict(ld_x=1 << 62)), (lin_call, dict(ld_y=1 << 62)),
])
def test_a_single_row_has_a_bounded_stride_too(call, bad):
    """2^62 elements of 4 bytes are 0 bytes in 64 bits, which no overlap check may divide by."""
    refused(call, rows=1, **bad)


MOST_COLS = 2 ** 31 - 1 - 16384   # column indices are 32 bits wide, and run past the row's end by what a workgroup takes at once


@pytest.mark.parametrize("cols", [MOST_COLS + 1, 2 ** 31 - 8193, 2 ** 31 - 1])
@pytest.mark.parametrize("rows", [0, 1])
def test_rows_too_long_for_their_indices_are_refused(cols, rows):
    far = {name: (i + 1) << 40 for i, name in enumerate(ADDR)}
    for call in (rows_call, norm_call):
        refused(call, rows=rows, cols=cols, **far)
        assert "cols" in aqd.last_error()


def test_the_longest_rows_are_taken():
    rows_call(rows=0, cols=MOST_COLS)
    norm_call(rows=0, cols=MOST_COLS)


@pytest.mark.parametrize("shape, parts, act", [
    (linear_plan.T64x64, 1, aqd.QLIN_SILU_GATE), (linear_plan.T64x64, 2, aqd.QLIN_SILU_GATE),   # plain only
    (linear_plan.FEW16, 2, aqd.QLIN_PLAIN), (linear_plan.FEW64, 2, aqd.QLIN_SILU_GATE),         # never split
    (len(linear_plan.NAMES), 1, aqd.QLIN_PLAIN), (-1, 1, aqd.QLIN_PLAIN),
])
def test_a_kernel_that_is_not_there_is_an_error(shape, parts, act):
    """A plan may name a kernel that has no such form: an error, where a launch of nothing would be a success."""
    for kind in (aqd.F32, aqd.F16, aqd.BF16):
        assert linear_plan.launch(linear_plan.args(64, 256, 4096, kind, act), (shape, parts, 0)) == 1   # hipErrorInvalidValue

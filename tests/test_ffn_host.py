"""Host logic of the gated feed-forward block (ffn.GatedFfn), without a GPU: the library's calls are
recorded, not run, so what the kernels would be given is checked on CPU tensors."""
import pytest
import torch

from paper_2007_06919_amd import aqd, ffn

HIDDEN, UNITS, ROWS = 64, 96, 4


@pytest.fixture
def calls(monkeypatch):
    """The library's calls in order, as (name, arguments)."""
    made = []
    for name in ("qrows_run", "qnorm_run", "qlin_run"):
        monkeypatch.setattr(aqd, name, lambda *a, _name=name, **kw: made.append((_name, a)))
    return made


def weights(dtype=torch.bfloat16):
    return tuple(torch.ones(*s, dtype=dtype) for s in ((HIDDEN,), (UNITS, HIDDEN), (UNITS, HIDDEN), (HIDDEN, UNITS)))


def rows_of(rows=ROWS, hidden=HIDDEN):
    return torch.zeros(rows, hidden, dtype=torch.bfloat16)


@pytest.mark.parametrize("default", [torch.bfloat16, torch.float16, torch.float64])
def test_scales_have_32_bits_whatever_the_default_type(calls, default):
    """The kernels write max_rows fp32 scales; a buffer of the default type would be half of that under 16 bits."""
    torch.set_default_dtype(default)
    try:
        f = ffn.GatedFfn(*weights(), max_rows=ROWS)
    finally:
        torch.set_default_dtype(torch.float32)
    for q in (f.q1, f.q2, f.s1, f.s2):
        assert q.dtype == torch.float32
    assert f.q1.shape == f.q2.shape == (ROWS,)

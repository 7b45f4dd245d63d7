"""The gated feed-forward block (ffn.GatedFfn) against its own steps in 64 bits, and its graph against eager passes.

The steps are taken on the codes and scales that the block itself made (their own tests hold them to their
definitions), so the tolerances are those of one product each: four roundings of fp32, the gate's
exponential, and one rounding to bf16 (2^-8 of the value)."""
import pytest

from paper_2007_06919_amd import aqd, ffn

pytestmark = pytest.mark.gpu


def block(torch, hidden, units, rows, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def randn(*shape, scale=1.0):
        return (torch.randn(*shape, generator=g, device="cuda") * scale).bfloat16()

    w = (1 + 0.1 * randn(hidden), randn(units, hidden, scale=hidden ** -0.5), randn(units, hidden, scale=hidden ** -0.5),
         randn(hidden, units, scale=units ** -0.5))
    return ffn.GatedFfn(*w, max_rows=rows), w, randn


@pytest.mark.parametrize("rows, hidden, units", [(1, 256, 640), (3, 250, 333), (40, 512, 1000), (300, 1024, 768)])
def test_block(rows, hidden, units):
    import torch
    f, w, randn = block(torch, hidden, units, rows)
    x, r = randn(rows, hidden), randn(rows, hidden)
    y, total = torch.empty_like(x), torch.empty_like(x)
    f.forward(x, r, y, total)
    torch.cuda.synchronize()
    assert torch.equal(total, (x.float() + r.float()).bfloat16())

    def product(c, q, w, s, k):
        return torch.mm(c[:, :k].double() * q.double()[:, None], (w.double() * s.double()[:, None]).t().contiguous())

    z = product(f.c1, f.q1, f.w1, f.s1, hidden)
    h = z[:, :units] * torch.sigmoid(z[:, :units]) * z[:, units:]
    tol = h.abs() * (2.0 ** -8 + 2.0 ** -18) + (z[:, units:].abs() + z[:, :units].abs()) * 2.0 ** -20
    assert bool(((f.h[:rows].double() - h).abs() <= tol).all())
    want = product(f.c2, f.q2, f.w2, f.s2, units)
    assert bool(((y.double() - want).abs() <= want.abs() * 2.0 ** -8 + want.abs().max() * 2.0 ** -20).all())
    # and near the block on the unquantised weights: codes of 8 bits are off by 1 part in 250 of the row's largest
    real = ffn.reference(x, r, *w, f.eps)
    assert float((y.float() - real).norm() / real.norm()) < 0.05


def test_graph_and_in_place_residual():
    import torch
    rows, hidden = 24, 768
    f, _, randn = block(torch, hidden, 1280, rows)
    stream = torch.cuda.Stream()
    x, r, y = randn(rows, hidden), randn(rows, hidden), torch.empty(rows, hidden, device="cuda").bfloat16()
    torch.cuda.synchronize()
    f.capture(x, r, y, r, stream)
    try:
        for _ in range(3):
            x.copy_(randn(rows, hidden))
            before, eager, total = r.clone(), torch.empty_like(y), torch.empty_like(r)
            f.forward(x, before, eager, total)
            torch.cuda.synchronize()
            f.replay(stream)
            torch.cuda.synchronize()
            assert torch.equal(y, eager) and torch.equal(r, total)
    finally:
        f.close()


def test_refusals():
    import torch
    f, w, randn = block(torch, 64, 96, 4)
    x = randn(4, 64)
    with pytest.raises(ValueError):
        ffn.GatedFfn(w[0], w[1], w[2], w[1])
    with pytest.raises(ValueError):
        ffn.GatedFfn(*w, max_rows=0)
    with pytest.raises(ValueError):
        f.forward(randn(5, 64), randn(5, 64), randn(5, 64), randn(5, 64))
    with pytest.raises(ValueError):
        f.forward(x, x.float(), x.clone(), x.clone())
    with pytest.raises(ValueError):
        f.forward(x, x.clone(), x.clone(), randn(64, 4).t())
    wider = randn(5, 64)
    with pytest.raises(aqd.AqdError):   # total is x, shifted by one element
        f.forward(wider[:4], x, x.clone(), wider.view(-1)[1:257].view(4, 64))


def test_under_a_16_bit_default_type():
    """torch's default type may be 16 bits wide, as in language-model programs: the block's scales stay fp32."""
    import torch
    rows, hidden, units = 40, 512, 1000
    outs = []
    for default in (torch.float32, torch.bfloat16):
        torch.set_default_dtype(default)
        try:
            g = torch.Generator(device="cuda").manual_seed(1)
            w = [torch.randn(*s, generator=g, device="cuda", dtype=torch.float32).bfloat16() / 16
                 for s in ((hidden,), (units, hidden), (units, hidden), (hidden, units))]
            x = torch.randn(2, rows, hidden, generator=g, device="cuda", dtype=torch.float32).bfloat16()
            f = ffn.GatedFfn(*w, max_rows=rows)
            assert f.q1.dtype == f.q2.dtype == torch.float32
            y, total = torch.empty_like(x[0]), torch.empty_like(x[0])
            f.forward(x[0], x[1], y, total)
            torch.cuda.synchronize()
        finally:
            torch.set_default_dtype(torch.float32)
        outs.append((y, total, f.q1.clone(), f.q2.clone()))
    for a, b in zip(*outs):
        assert torch.equal(a, b)
    assert outs[0][0].ne(0).any()


def test_without_a_residual():
    """The first block of a network: the same as a residual of zeros, with the sum asked for and without."""
    import torch
    rows, hidden = 7, 256
    f, _, randn = block(torch, hidden, 640, rows)
    x = randn(rows, hidden)
    y, total = [torch.empty_like(x) for _ in range(3)], [torch.empty_like(x) for _ in range(2)]
    f.forward(x, torch.zeros_like(x), y[0], total[0])
    f.forward(x, None, y[1], total[1])
    f.forward(x, None, y[2], None)
    torch.cuda.synchronize()
    assert torch.equal(y[0], y[1]) and torch.equal(y[0], y[2]) and y[0].ne(0).any()
    assert torch.equal(total[0], x) and torch.equal(total[1], x)


def test_matrices_of_any_strides():
    """Weights handed over as transposed, sliced or expanded views give the codes of their packed copies."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(3)
    wide = torch.randn(48, 96, generator=g, device="cuda")
    for m in (wide, wide[:, ::2], wide.t(), wide[:1].expand(5, 96), wide[:1, ::3], wide[:, 3:30]):
        codes, scales = ffn.quantize_rows(m)
        want, want_scales = ffn.quantize_rows(m.clone(memory_format=torch.contiguous_format))
        assert torch.equal(codes, want) and torch.equal(scales, want_scales) and codes.shape == m.shape
        assert bool(((codes * scales[:, None] - m).abs() <= 0.51 * scales[:, None]).all())


def test_quantising_on_another_stream():
    """In order with the current stream on both sides, for a stream object and for its handle."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(6)
    w = torch.randn(2000, 1003, generator=g, device="cuda")
    want = ffn.quantize_rows(w)
    side = torch.cuda.Stream()
    for stream in (side, side.cuda_stream):
        fresh = w * 2 / 2   # on the current stream, not waited for
        codes, scales = ffn.quantize_rows(fresh, stream)
        got = codes.clone(), scales.clone()
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_first_pass_on_another_stream():
    """No wait between the set-up on the current stream and a pass on another one, nor before the block is dropped."""
    import torch
    rows, hidden = 16, 512
    f, w, randn = block(torch, hidden, 1024, rows)
    x, r = randn(rows, hidden), randn(rows, hidden)
    want, total = torch.empty_like(x), torch.empty_like(x)
    f.forward(x, r, want, total)
    torch.cuda.synchronize()
    side, y = torch.cuda.Stream(), torch.empty_like(x)
    g = ffn.GatedFfn(*w, max_rows=rows)
    g.forward(x, r, y, total, side)
    del g
    junk = [torch.full((1 << 20,), 77, dtype=torch.uint8, device="cuda") for _ in range(4)]
    torch.cuda.synchronize()
    assert torch.equal(y, want) and junk[0][0] == 77

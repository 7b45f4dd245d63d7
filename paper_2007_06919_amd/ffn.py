"""A gated feed-forward block on 8-bit weights, the four launches that serve it:

    sum, codes, scales = qnorm(x + residual)              residual's addition, norm, 8-bit codes
    h                  = qlin(codes, gate and up rows)    silu(gate) * up in the product's epilogue
    codes, scales      = qrows(h)                         8-bit codes of the hidden units
    y                  = qlin(codes, down rows)

Weights are quantised once, one scale per output channel, by the same row quantisation
that makes the activations' codes. All buffers are allocated at set-up for the most
rows of a call, so a pass allocates nothing and can be captured in a HIP graph
(``capture``, ``replay``). PyTorch provides device memory and the stream; all
arithmetic is in ``libaqd.so``.

    python -m paper_2007_06919_amd.ffn [hidden] [units]

times a block of random weights at 1 to 4096 rows, eager and replayed, and prints how
far its outputs are from the same block in fp32 on the unquantised weights.
"""
from __future__ import annotations

import sys

from . import aqd

DEVICE = "cuda"   # where the library's kernels run: no other address may reach them


def _meet(a, ld_a, b, ld_b, rows, cols):
    """Whether two [rows][cols] tensors of one type may share an element (column ranges of one buffer do not)."""
    if not rows:
        return False
    gap = (b.data_ptr() - a.data_ptr()) // a.element_size()
    if gap >= (rows - 1) * ld_a + cols or -gap >= (rows - 1) * ld_b + cols:
        return False
    return rows == 1 or ld_a != ld_b or gap % ld_a < cols or gap % ld_a + cols > ld_a


def quantize_rows(w, stream=None):
    """(codes, scales) of a real matrix, one scale per row; rows of codes start at multiples of 16 bytes. On `stream`
    (None: the current one) in order with the current stream: after the work that it has, before what it gets next."""
    import torch
    if w.device.type != DEVICE:
        raise ValueError(f"the matrix is on {w.device}, not on the GPU")
    if w.device.index is not None and w.device.index != torch.cuda.current_device():
        with torch.cuda.device(w.device.index):
            return quantize_rows(w, stream)
    rows, cols = w.shape
    if w.stride(1) != 1 or rows > 1 and w.stride(0) < cols:
        w = w.contiguous()
    codes = torch.empty(rows, -(-cols // 16) * 16, dtype=torch.int8, device=w.device)[:, :cols]
    scales = torch.empty(rows, dtype=torch.float32, device=w.device)
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(stream) if stream else torch.cuda.default_stream()
    if stream is not None:
        stream.wait_stream(torch.cuda.current_stream())
    aqd.qrows_run(rows, cols, aqd.real_type(w), w, w.stride(0) if rows > 1 else 0, codes, codes.stride(0), scales, stream)
    if stream is not None:
        torch.cuda.current_stream().wait_stream(stream)
    return codes, scales


def _finish(device, all=False):
    """Wait for the current stream, or for all."""
    import torch
    torch.cuda.synchronize(device) if all else torch.cuda.current_stream(device).synchronize()


def _streams_of(device):
    """Handles of the streams for which torch keeps tensors that are made now on `device` anyway: its current one, where the device is the
    current one too (the default streams of two devices have one handle)."""
    import torch
    return {aqd._stream(None)} if device.index is None or device.index == torch.cuda.current_device() else set()


class GatedFfn:
    """norm_weight [hidden], gate and up [units][hidden], down [hidden][units]: device tensors of one real type, that of
    the block's inputs and outputs too. The set-up has ended on the GPU when the constructor returns, so passes may run on any
    stream, one at a time. Before a block that ran on a stream given by its handle is dropped, that stream is waited for; those
    given as torch's streams, or current, torch waits for itself before it gives the block's memory to others."""

    def __init__(self, norm_weight, gate, up, down, eps=1e-5, max_rows=4096):
        import torch
        units, hidden = gate.shape
        if up.shape != gate.shape or down.shape != (hidden, units) or norm_weight.shape != (hidden,):
            raise ValueError(f"shapes do not make a block: norm {tuple(norm_weight.shape)}, gate {tuple(gate.shape)}, "
                             f"up {tuple(up.shape)}, down {tuple(down.shape)}")
        if not norm_weight.dtype == gate.dtype == up.dtype == down.dtype:
            raise ValueError(f"one type for all: norm {norm_weight.dtype}, gate {gate.dtype}, up {up.dtype}, down {down.dtype}")
        if gate.device.type != DEVICE or not norm_weight.device == gate.device == up.device == down.device:
            raise ValueError(f"one GPU for all: norm on {norm_weight.device}, gate on {gate.device}, up on {up.device}, "
                             f"down on {down.device}")
        if max_rows < 1:
            raise ValueError("max_rows must be at least 1")
        self.hidden, self.units, self.eps, self.max_rows = hidden, units, float(eps), max_rows
        self.dtype, self.type = gate.dtype, aqd.real_type(gate)
        self.norm_weight = norm_weight.contiguous()
        self.w1, self.s1 = quantize_rows(torch.cat([gate, up]))
        self.w2, self.s2 = quantize_rows(down)
        dev = self.device = gate.device
        self.index = dev.index

        def codes(cols):
            return torch.empty(max_rows, -(-cols // 16) * 16, dtype=torch.int8, device=dev)

        def scales():   # fp32 whatever torch's default type
            return torch.empty(max_rows, dtype=torch.float32, device=dev)

        self.c1, self.q1 = codes(hidden), scales()
        self.h = torch.empty(max_rows, units, dtype=self.dtype, device=dev)
        self.c2, self.q2 = codes(units), scales()
        # the bound serves every call; the block's launches follow one another on one stream
        self.ws_bytes = aqd.QLIN_WORKSPACE_BYTES
        self.workspace = torch.empty(self.ws_bytes, dtype=torch.uint8, device=dev)
        self.ld_c1, self.ld_w1, self.ld_c2, self.ld_w2 = (t.stride(0) for t in (self.c1, self.w1, self.c2, self.w2))
        self._graph = self._recorded = None
        self._buffers = (self.norm_weight, self.w1, self.s1, self.w2, self.s2, self.c1, self.q1, self.h, self.c2, self.q2,
                         self.workspace)
        self._streams = _streams_of(dev)   # handles of those that torch keeps the buffers for
        _finish(dev)

    def _use_on(self, stream):
        """The handle of `stream` (None: the current one), for which torch keeps the buffers from now on."""
        handle = aqd._stream(stream)
        if handle not in self._streams:
            import torch
            if stream is None:
                stream = torch.cuda.current_stream()
            if isinstance(stream, torch.cuda.Stream) and not isinstance(stream, torch.cuda.ExternalStream):
                for t in self._buffers:
                    t.record_stream(stream)
                self._streams.add(handle)
        return handle

    def forward(self, x, residual, y, total, stream=None):
        """y = block(norm(x + residual)), total = x + residual; all [rows][hidden] with contiguous rows that share no
        element (no expanded tensors). residual and total may be None (the first block of a network has no residual); total
        may be residual, and y may be x or residual, but not share an element with total. The tensors are ready on `stream` (None: the
        current one) and outlive the pass. On one stream at a time."""
        import torch
        if self.index is not None and self.index != torch.cuda.current_device():
            with torch.cuda.device(self.index):
                return self.forward(x, residual, y, total, stream)
        rows, hidden, units, ws = x.shape[0], self.hidden, self.units, self.workspace
        if rows > self.max_rows:
            raise ValueError(f"{rows} rows, and buffers for {self.max_rows}")
        ld_x, ld_y = self._row_stride(x, rows), self._row_stride(y, rows)
        ld_residual = 0 if residual is None else self._row_stride(residual, rows)
        ld_total = 0 if total is None else self._row_stride(total, rows)
        if total is not None and _meet(y, ld_y, total, ld_total, rows, hidden):
            raise ValueError("y and total share memory")
        stream = self._use_on(stream)
        aqd.qnorm_run(rows, hidden, self.type, self.eps, x, ld_x, residual, ld_residual, self.norm_weight, total, ld_total,
                      self.c1, self.ld_c1, self.q1, stream)
        aqd.qlin_run(rows, units, hidden, self.type, aqd.QLIN_SILU_GATE, self.c1, self.ld_c1, self.q1, self.w1, self.ld_w1, self.s1, None,
                     self.h, units, ws, self.ws_bytes, stream)
        aqd.qrows_run(rows, units, self.type, self.h, units, self.c2, self.ld_c2, self.q2, stream)
        aqd.qlin_run(rows, hidden, units, self.type, aqd.QLIN_PLAIN, self.c2, self.ld_c2, self.q2, self.w2, self.ld_w2, self.s2, None,
                     y, ld_y, ws, self.ws_bytes, stream)
        return y

    def _row_stride(self, t, rows):
        """A caller's tensor, checked; its row stride as the library takes it, which reads 0 as packed rows. A single row has none."""
        if t.shape != (rows, self.hidden) or t.dtype != self.dtype or t.device != self.device:
            raise ValueError(f"tensors must be [{rows}][{self.hidden}] {self.dtype} on {self.device}")
        ld, step = t.stride()
        if step != 1:
            raise ValueError("the rows of a tensor are not contiguous")
        if rows < 2:
            return 0
        if ld < self.hidden:
            raise ValueError(f"rows of a tensor share memory: {self.hidden} columns, stride {ld}")
        return ld

    def capture(self, x, residual, y, total, stream):
        """Record a pass on these tensors into a HIP graph (`stream`: not the null stream), which holds them until `close` or
        the next recording."""
        self.close()
        aqd.graph_begin(stream)
        try:
            self.forward(x, residual, y, total, stream)
        except BaseException:
            try:
                aqd.graph_destroy(aqd.graph_end(stream))
            except aqd.AqdError:
                pass
            raise
        self._graph = aqd.graph_end(stream)
        self._recorded = x, residual, y, total

    def replay(self, stream):
        if self._graph is None:
            raise RuntimeError("no pass is recorded: capture() first")
        import torch
        if self.index is not None and self.index != torch.cuda.current_device():
            with torch.cuda.device(self.index):
                return self.replay(stream)
        aqd.graph_launch(self._graph, self._use_on(stream))

    def close(self):
        """Forget the recorded pass."""
        if self._graph is not None:
            _finish(self.device, all=True)   # no replay may be pending
            aqd.graph_destroy(self._graph)
            self._graph = self._recorded = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def reference(x, residual, norm_weight, gate, up, down, eps):
    """The block in fp32 on the unquantised weights."""
    import torch
    s = x.float() + residual.float()
    n = s * torch.rsqrt((s * s).mean(1, keepdim=True) + eps) * norm_weight.float()
    g = n @ gate.float().t()
    return (g * torch.sigmoid(g) * (n @ up.float().t())) @ down.float().t()


def main(hidden=4096, units=11264):
    import torch
    g = torch.Generator(device="cuda").manual_seed(0)

    def randn(*shape, scale=1.0):
        return (torch.randn(*shape, generator=g, device="cuda") * scale).bfloat16()

    w = (1 + 0.1 * randn(hidden), randn(units, hidden, scale=hidden ** -0.5), randn(units, hidden, scale=hidden ** -0.5),
         randn(hidden, units, scale=units ** -0.5))
    ffn = GatedFfn(*w)
    stream = torch.cuda.Stream()
    for rows in (1, 16, 128, 1024, 4096):
        x, r = randn(rows, hidden), randn(rows, hidden)
        y, total = torch.empty_like(x), torch.empty_like(x)
        torch.cuda.synchronize()
        ffn.forward(x, r, y, total, stream)
        torch.cuda.synchronize()
        want = reference(x, r, *w, ffn.eps)
        off = float((y.float() - want).norm() / want.norm())
        ffn.capture(x, r, y, total, stream)
        line = f"{rows:5d} rows: {100 * off:.2f}% off fp32"
        ops = 6 * rows * hidden * units
        for name, run in (("eager", lambda: ffn.forward(x, r, y, total, stream)), ("replayed", lambda: ffn.replay(stream))):
            for _ in range(10):
                run()
            begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            begin.record(stream)
            for _ in range(50):
                run()
            end.record(stream)
            torch.cuda.synchronize()
            us = begin.elapsed_time(end) / 50 * 1e3
            line += f", {name} {us:.1f} us ({ops / us / 1e6:.0f} TOPS)"
        print(line, flush=True)
    ffn.close()


if __name__ == "__main__":
    main(*(int(a) for a in sys.argv[1:3]))

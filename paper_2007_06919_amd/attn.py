"""An attention block on 8-bit weights with a cache of keys and values in 4 bits, the launches that serve it:

    total, codes, scales = qnorm(x + residual)            residual's addition, norm, 8-bit codes
    qkv                  = qlin(codes)                    queries, keys and values in one product
    q, k                 = heads(q, k)                    norms of the heads, rotation by position, in place
    cache                = qcache_write(k, v)             4-bit codes into the sequences' pages
    h                    = attn(q, k, v) or qattn(q, cache)   where all sequences are new, or some of them are in the cache
    codes, scales        = qrows(h)
    y                    = qlin(codes)

In float16 and bfloat16 it takes and gives what the feed-forward block of ``ffn.py`` does, so the two make a layer. ``PagedCache`` keeps which
pages a sequence has; one of its steps (``Step``) serves every layer that has a cache of its shape. PyTorch provides
device memory and the stream; all arithmetic is in ``libaqd.so``.

    python -m paper_2007_06919_amd.attn [hidden] [q_heads] [heads] [dim]

times a block of random weights on prompts and on single tokens of 1 to 64 sequences, and prints how far its outputs are from
the same block in fp32 on unquantised weights and cache.
"""
from __future__ import annotations

import sys

from . import aqd
from .ffn import DEVICE, _finish, _meet, _streams_of, quantize_rows


class Step:
    """The tokens that one pass works on: `counts` new tokens of each sequence, as rows behind one another. Index tensors on
    the device, which a pass reads when it runs; they are ready on every stream."""

    def __init__(self, cache, ids, counts):
        import torch
        self.cache, self.ids, self.counts = cache, tuple(ids), tuple(counts)
        before = [cache.lengths[i] for i in ids]
        after = [a + n for a, n in zip(before, counts)]
        self.rows, self.batch = sum(counts), len(ids)
        self.max_queries, self.max_keys = max(counts, default=0), max(after, default=0)
        # keys and values of whole prompts are those of the pass itself
        self.prompts = not any(before)
        width = max((len(cache.pages_of[i]) for i in ids), default=0)
        self.ld_table = max(width, 1)
        position, slots, start, tables = [], [], [0], []
        for i, a, n in zip(ids, before, counts):
            pages = cache.pages_of[i]
            position += range(a, a + n)
            slots += [pages[t // cache.page] * cache.page + t % cache.page for t in range(a, a + n)]
            start.append(start[-1] + n)
            tables += pages + [0] * (self.ld_table - len(pages))

        def put(values):
            return torch.tensor(values, dtype=torch.int32, device=cache.device)

        self.tensors = tuple(put(v) for v in (position, slots, start, after, tables))
        self.position, self.slots, self.start, self.lengths, self.tables = self.tensors
        self.streams = _streams_of(cache.device)   # handles of those that torch keeps the tensors for
        _finish(cache.device)


class PagedCache:
    """Which pages of `page` tokens, of `pages` that there are, each sequence has. `layer()` makes a layer's cache."""

    def __init__(self, heads, dim, pages, group=32, page=64, device=None):
        import torch
        self.heads, self.dim, self.group, self.page, self.pages = heads, dim, group, page, pages
        self.desc = aqd.QcacheDesc(heads, dim, group, page, pages)
        self.bytes = aqd.qcache_bytes(self.desc)     # checks the shape
        self.device = torch.empty(0, device=device or DEVICE).device   # with its index
        if self.device.type != DEVICE:
            raise ValueError(f"the cache is on {self.device}, not on the GPU")
        self.free = list(range(pages - 1, -1, -1))
        self.pages_of, self.lengths, self._next = {}, {}, 0

    def layer(self):
        """Memory of one layer's cache."""
        import torch
        return torch.zeros(self.bytes, dtype=torch.uint8, device=self.device)

    def add(self):
        """A new, empty sequence's number."""
        i = self._next
        self._next += 1
        self.pages_of[i], self.lengths[i] = [], 0
        return i

    def remove(self, i):
        """Gives a sequence's pages back. Passes that read them have ended, or are on the stream of those that come next."""
        self.free += reversed(self.pages_of.pop(i))
        del self.lengths[i]

    def shorten(self, i, length):
        """Takes a sequence's tokens from `length` on back (drafts that were refused, a step whose pass failed), and the pages that only
        they had. Steps of those tokens have no more passes; as for `remove`, passes that read their pages have ended."""
        if not 0 <= length <= self.lengths[i]:
            raise ValueError(f"a sequence of {self.lengths[i]} tokens cannot be shortened to {length}")
        pages, keep = self.pages_of[i], -(-length // self.page)
        self.free += reversed(pages[keep:])
        del pages[keep:]
        self.lengths[i] = length

    def step(self, ids, counts):
        """A Step of counts[j] new tokens of sequence ids[j]; takes the pages that they need. The tokens belong to their sequences from
        now on (until `shorten` takes them back): every layer's pass of this step comes before the next step's."""
        ids, counts = list(ids), [int(n) for n in counts]
        if len(ids) != len(counts) or len(set(ids)) != len(ids) or any(i not in self.lengths for i in ids):
            raise ValueError("a step names sequences of the cache, each once, and a count for each")
        if any(n < 0 for n in counts):
            raise ValueError("a count is negative")
        need = [max(0, -(-(self.lengths[i] + n) // self.page) - len(self.pages_of[i])) for i, n in zip(ids, counts)]
        if sum(need) > len(self.free):
            raise MemoryError(f"{sum(need)} pages are needed, {len(self.free)} are free")
        for i, n in zip(ids, need):
            self.pages_of[i] += [self.free.pop() for _ in range(n)]
        step = Step(self, ids, counts)
        for i, n in zip(ids, counts):
            self.lengths[i] += n
        return step


class CachedAttention:
    """norm_weight [hidden], wq [q_heads * dim][hidden], wk and wv [heads * dim][hidden], wo [hidden][q_heads * dim], q_norm and
    k_norm [dim] or None: device tensors of one real type, float16 or bfloat16, that of the block's inputs and outputs too. table:
    cosines and sines [positions][rot] (aqd.h; rotary_table). cache: the PagedCache whose steps it takes. The set-up has ended on the
    GPU when the constructor returns, so passes may run on any stream, one at a time (see GatedFfn). A step of new sequences alone attends
    to its own keys and values; where others are among them, all of its rows go through the cache and have its 4 bits' error."""

    def __init__(self, cache, norm_weight, wq, wk, wv, wo, table, q_norm=None, k_norm=None, pairs=aqd.PAIRS_HALVES, eps=1e-5, max_rows=4096):
        import torch
        heads, dim = cache.heads, cache.dim
        wide, hidden = wq.shape
        if wide % dim or (wide // dim) % heads or wk.shape != (heads * dim, hidden) or wv.shape != wk.shape or wo.shape != (hidden, wide) or \
                norm_weight.shape != (hidden,) or any(w is not None and w.shape != (dim,) for w in (q_norm, k_norm)):
            raise ValueError(f"shapes do not make a block of {heads} key heads of {dim}: norm {tuple(norm_weight.shape)}, wq {tuple(wq.shape)}, "
                             f"wk {tuple(wk.shape)}, wv {tuple(wv.shape)}, wo {tuple(wo.shape)}")
        given = [t for t in (norm_weight, wq, wk, wv, wo, q_norm, k_norm) if t is not None]
        if any(t.dtype != wq.dtype for t in given) or wq.dtype not in (torch.float16, torch.bfloat16):
            raise ValueError(f"one type for all, float16 or bfloat16: {[str(t.dtype) for t in given]}")
        if any(t.device != cache.device for t in given + [table]):
            raise ValueError(f"one GPU for all: the cache is on {cache.device}, others on {[str(t.device) for t in given + [table]]}")
        if table.dtype != torch.float32 or table.dim() != 2 or table.shape[1] % 2 or table.shape[1] > dim:
            raise ValueError(f"the table must be float32 [positions][rot], rot even and at most {dim}: {table.dtype} {tuple(table.shape)}")
        if max_rows < 1:
            raise ValueError("max_rows must be at least 1")
        self.cache, self.hidden, self.q_heads, self.heads, self.dim = cache, hidden, wide // dim, heads, dim
        self.eps, self.pairs, self.max_rows = float(eps), pairs, max_rows
        self.dtype, self.type, self.device, self.index = wq.dtype, aqd.real_type(wq), cache.device, cache.device.index
        self.norm_weight, self.table = norm_weight.contiguous(), table.contiguous()
        self.q_norm, self.k_norm = [None if w is None else w.contiguous() for w in (q_norm, k_norm)]
        self.w1, self.s1 = quantize_rows(torch.cat([wq, wk, wv]))
        self.w2, self.s2 = quantize_rows(wo)
        self.data = cache.layer()
        dev, self.wide = self.device, wide + 2 * heads * dim

        def codes(cols):
            return torch.empty(max_rows, -(-cols // 16) * 16, dtype=torch.int8, device=dev)

        def scales():   # fp32 whatever torch's default type
            return torch.empty(max_rows, dtype=torch.float32, device=dev)

        self.c1, self.q1, self.c2, self.q2 = codes(hidden), scales(), codes(wide), scales()
        self.qkv = torch.empty(max_rows, self.wide, dtype=self.dtype, device=dev)
        self.h = torch.empty(max_rows, wide, dtype=self.dtype, device=dev)
        # one bound serves every call of either kind; the block's launches follow one another on one stream
        self.ws_bytes = max(aqd.QLIN_WORKSPACE_BYTES, aqd.ATTN_WORKSPACE_BYTES)
        self.workspace = torch.empty(self.ws_bytes, dtype=torch.uint8, device=dev)
        self._buffers = (self.norm_weight, self.table, self.w1, self.s1, self.w2, self.s2, self.data, self.c1, self.q1, self.c2, self.q2,
                         self.qkv, self.h, self.workspace) + tuple(w for w in (self.q_norm, self.k_norm) if w is not None)
        self._streams = _streams_of(dev)   # handles of those that torch keeps the buffers for
        _finish(dev)

    def forward(self, x, residual, y, total, step, stream=None):
        """y = block(norm(x + residual)), total = x + residual, of the tokens of `step`: [rows][hidden] each, as GatedFfn's. residual
        and total may be None. Writes the tokens' keys and values into the layer's cache first, so a token sees itself."""
        import torch
        if self.index is not None and self.index != torch.cuda.current_device():
            with torch.cuda.device(self.index):
                return self.forward(x, residual, y, total, step, stream)
        if step.cache is not self.cache:
            raise ValueError("the step is of another cache")
        rows, hidden, dim, wide = step.rows, self.hidden, self.dim, self.wide
        if rows > self.max_rows:
            raise ValueError(f"{rows} rows, and buffers for {self.max_rows}")
        if step.max_keys > self.table.shape[0]:
            raise ValueError(f"{step.max_keys} positions, and a table of {self.table.shape[0]}")
        ld_x, ld_y = self._row_stride(x, rows), self._row_stride(y, rows)
        ld_residual = 0 if residual is None else self._row_stride(residual, rows)
        ld_total = 0 if total is None else self._row_stride(total, rows)
        if total is not None and _meet(y, ld_y, total, ld_total, rows, hidden):
            raise ValueError("y and total share memory")
        stream = self._use_on(stream, step)
        at_k, at_v = self.q_heads * dim, (self.q_heads + self.heads) * dim
        q, k, v = self.qkv, self.qkv[:, at_k:], self.qkv[:, at_v:]
        ws, ws_bytes = self.workspace, self.ws_bytes
        aqd.qnorm_run(rows, hidden, self.type, self.eps, x, ld_x, residual, ld_residual, self.norm_weight, total, ld_total,
                      self.c1, self.c1.stride(0), self.q1, stream)
        aqd.qlin_run(rows, wide, hidden, self.type, aqd.QLIN_PLAIN, self.c1, self.c1.stride(0), self.q1, self.w1, self.w1.stride(0), self.s1, None,
                     q, wide, ws, ws_bytes, stream)
        aqd.heads_run(rows, self.q_heads, self.heads, dim, self.table.shape[1], self.pairs, self.type, self.table.shape[0], self.eps,
                      q, wide, dim, k, wide, dim, self.q_norm, self.k_norm, step.position, self.table, q, wide, dim, k, wide, dim, stream)
        aqd.qcache_write(self.cache.desc, rows, self.type, k, wide, dim, v, wide, dim, step.slots, self.data, stream)
        if step.prompts:
            aqd.attn_run(step.batch, self.q_heads, self.heads, dim, rows, rows, step.max_queries, step.max_keys, True, self.type, dim ** -0.5,
                         q, wide, dim, k, wide, dim, v, wide, dim, step.start, step.start, self.h, at_k, dim, ws, ws_bytes, stream)
        else:
            aqd.qattn_run(self.cache.desc, step.batch, self.q_heads, rows, step.max_queries, step.max_keys, self.type, dim ** -0.5,
                          q, wide, dim, step.start, self.data, step.tables, step.ld_table, step.lengths, self.h, at_k, dim, ws, ws_bytes, stream)
        aqd.qrows_run(rows, at_k, self.type, self.h, at_k, self.c2, self.c2.stride(0), self.q2, stream)
        aqd.qlin_run(rows, hidden, at_k, self.type, aqd.QLIN_PLAIN, self.c2, self.c2.stride(0), self.q2, self.w2, self.w2.stride(0), self.s2, None,
                     y, ld_y, ws, ws_bytes, stream)
        return y

    def _use_on(self, stream, step):
        """The handle of `stream` (None: the current one), for which torch keeps the block's buffers and the step's from now on."""
        handle = aqd._stream(stream)
        for known, tensors in ((self._streams, self._buffers), (step.streams, step.tensors)):
            if handle not in known:
                import torch
                if stream is None:
                    stream = torch.cuda.current_stream()
                if isinstance(stream, torch.cuda.Stream) and not isinstance(stream, torch.cuda.ExternalStream):
                    for t in tensors:
                        t.record_stream(stream)
                    known.add(handle)
        return handle

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


def rotary_table(positions, rot, base=10000.0, device=None):
    """Cosines and sines [positions][rot] of angles position * base^(-2 i / rot), computed in 64 bits."""
    import torch
    device = device or DEVICE
    f = float(base) ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=device) / rot)
    a = torch.arange(positions, dtype=torch.float64, device=device)[:, None] * f
    return torch.cat([a.cos(), a.sin()], 1).float().contiguous()


def reference(x, residual, norm_weight, wq, wk, wv, wo, table, q_norm, k_norm, eps, heads, dim):
    """The block in fp32 on the unquantised weights, of one whole sequence x [tokens][hidden] (halves rotated)."""
    import torch
    s = x.float() + residual.float()
    n = s * torch.rsqrt((s * s).mean(1, keepdim=True) + eps) * norm_weight.float()
    tokens, rot = len(x), table.shape[1]

    def turned(w, weight):
        t = (n @ w.float().t()).unflatten(1, (-1, dim))
        if weight is not None:
            t = t * torch.rsqrt((t * t).mean(2, keepdim=True) + eps) * weight.float()
        c, d = table[:tokens, None, :rot // 2], table[:tokens, None, rot // 2:]
        a, b = t[..., :rot // 2], t[..., rot // 2:rot]
        return torch.cat([a * c - b * d, b * c + a * d, t[..., rot:]], 2)

    q, k, v = turned(wq, q_norm), turned(wk, k_norm), (n @ wv.float().t()).unflatten(1, (-1, dim))
    h = torch.empty_like(q)
    hidden = torch.ones(tokens, tokens, dtype=torch.bool, device=x.device).triu(1)
    per = q.shape[1] // heads
    for i in range(q.shape[1]):
        p = (q[:, i] @ k[:, i // per].t().contiguous()) * dim ** -0.5
        h[:, i] = torch.softmax(p.masked_fill(hidden, float("-inf")), 1) @ v[:, i // per].contiguous()
    return h.flatten(1) @ wo.float().t()


def main(hidden=4096, q_heads=32, heads=8, dim=128):
    import torch
    g = torch.Generator(device=DEVICE).manual_seed(0)

    def randn(*shape, scale=1.0):
        return (torch.randn(*shape, generator=g, device=DEVICE) * scale).bfloat16()

    w = dict(norm_weight=1 + 0.1 * randn(hidden), wq=randn(q_heads * dim, hidden, scale=hidden ** -0.5), wk=randn(heads * dim, hidden, scale=hidden ** -0.5),
             wv=randn(heads * dim, hidden, scale=hidden ** -0.5), wo=randn(hidden, q_heads * dim, scale=(q_heads * dim) ** -0.5),
             table=rotary_table(8192, dim), q_norm=1 + 0.1 * randn(dim), k_norm=1 + 0.1 * randn(dim))
    cache = PagedCache(heads, dim, pages=64 * 65)
    block = CachedAttention(cache, max_rows=4096, **w)

    def timed(name, run):
        for _ in range(5):
            run()
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        begin.record()
        for _ in range(30):
            run()
        end.record()
        torch.cuda.synchronize()
        print(f"{name}: {begin.elapsed_time(end) / 30 * 1e3:.1f} us", flush=True)

    # a prompt, then its last tokens one by one from the cache: both against the same sequence in fp32
    x, r = randn(600, hidden), randn(600, hidden)
    y, total = torch.empty_like(x), torch.empty_like(x)
    one = cache.add()
    block.forward(x[:590], r[:590], y[:590], total[:590], cache.step([one], [590]))
    for t in range(590, 600):
        block.forward(x[t:t + 1], r[t:t + 1], y[t:t + 1], total[t:t + 1], cache.step([one], [1]))
    want = reference(x, r, eps=block.eps, heads=heads, dim=dim, **w)
    for name, rows in (("prompt", slice(0, 590)), ("single tokens", slice(590, 600))):
        print(f"{name}: {100 * float((y[rows].float() - want[rows]).norm() / want[rows].norm()):.2f}% off fp32", flush=True)
    cache.remove(one)
    for batch, each in ((1, 4000), (16, 4000), (64, 4000)):
        ids = [cache.add() for _ in range(batch)]
        x = randn(4000, hidden)
        y = torch.empty_like(x)
        for i in ids:
            step = cache.step([i], [each])
            block.forward(x, None, y, None, step)
        if batch == 1:
            timed(f"prompt of {each}", lambda: block.forward(x, None, y, None, step))
        step = cache.step(ids, [1] * batch)
        timed(f"a token of {batch} sequences of {each}", lambda: block.forward(x[:batch], None, y[:batch], None, step))
        for i in ids:
            cache.remove(i)


if __name__ == "__main__":
    main(*(int(a) for a in sys.argv[1:5]))

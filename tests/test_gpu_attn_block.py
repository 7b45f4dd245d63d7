"""The attention block (attn.CachedAttention) on the GPU: each of its steps against 64 bits on what the step before left, prompts
and single tokens; the whole against fp32; other streams; a recorded step.

The steps' tolerances are those of their operators (test_gpu_linear.py, test_gpu_attention.py), on the block's own buffers:
products are four roundings of fp32 and one to T (half the smallest number of T below its normal ones); heads: the products' rounding to T enters the norm twice, u(T) of the
element and of the norm."""
import numpy as np
import pytest

import attention_plain as plain
from attention_plain import DTYPE, HALF, LEAST
from paper_2007_06919_amd import aqd, attn
from test_gpu_attention import OFFSET, U, check_attention, close

pytestmark = pytest.mark.gpu
HIDDEN, Q_HEADS, HEADS, DIM = 256, 6, 2, 64


def make(torch, t, norms=True, seed=0, rot=32, group=32, page=16, pages=40):
    rng = np.random.Generator(np.random.PCG64(seed))

    def w(*shape, scale):
        return torch.from_numpy(rng.standard_normal(shape) * scale).to(DTYPE[t]).cuda()

    weights = dict(norm_weight=1 + w(HIDDEN, scale=0.1), wq=w(Q_HEADS * DIM, HIDDEN, scale=HIDDEN ** -0.5), wk=w(HEADS * DIM, HIDDEN, scale=HIDDEN ** -0.5),
                   wv=w(HEADS * DIM, HIDDEN, scale=HIDDEN ** -0.5), wo=w(HIDDEN, Q_HEADS * DIM, scale=(Q_HEADS * DIM) ** -0.5),
                   table=attn.rotary_table(500, rot), q_norm=1 + w(DIM, scale=0.2) if norms else None, k_norm=1 + w(DIM, scale=0.2) if norms else None)
    cache = attn.PagedCache(HEADS, DIM, pages, group=group, page=page)
    return rng, w, weights, cache, attn.CachedAttention(cache, max_rows=300, **weights)


def product(codes, scales, rows, weights, weight_scales, outs, cols):
    """Whole numbers' sums, then the scales: a sum of 0 is 0."""
    x, w = codes[:rows, :cols].double().cpu().numpy(), weights[:outs, :cols].double().cpu().numpy()
    return (x @ w.T) * scales[:rows].double().cpu().numpy()[:, None] * weight_scales[:outs].double().cpu().numpy()


def check_pass(torch, block, weights, step, y, t, before):
    """Every step of the pass that `step` was, on the block's buffers. before: the cache's bytes before it."""
    rows, wide = step.rows, block.wide
    host = [v.cpu().numpy() for v in (step.position, step.slots, step.start, step.lengths, step.tables)]
    position, slots, start, lengths, tables = host
    # joint projection, norms, rotation: in place in one buffer
    z = product(block.c1, block.q1, rows, block.w1, block.s1, wide, HIDDEN).reshape(rows, -1, DIM)
    got = block.qkv[:rows].double().cpu().numpy().reshape(rows, -1, DIM)
    table = weights["table"].double().cpu().numpy()
    ends = ((0, Q_HEADS, weights["q_norm"]), (Q_HEADS, Q_HEADS + HEADS, weights["k_norm"]))
    for a, b, norm in ends:
        n = None if norm is None else norm.double().cpu().numpy()
        want, size = plain.heads(z[:, a:b], n, block.eps, table, position, table.shape[1], True)
        close(got[:, a:b], want, (2 * HALF[t] + 30 * U) * size + HALF[t] * np.abs(want) * 1.01 + LEAST[t], "heads")
    v = z[:, Q_HEADS + HEADS:]
    close(got[:, Q_HEADS + HEADS:], v, 4 * U * np.abs(v) + HALF[t] * np.abs(v) * 1.01 + LEAST[t], "values")
    # the cache
    c = block.cache
    cache = before.copy()
    plain.write(cache, slots, got[:, Q_HEADS:Q_HEADS + HEADS].astype(np.float32), got[:, Q_HEADS + HEADS:].astype(np.float32), HEADS, DIM, c.group, c.page)
    assert np.array_equal(block.data.cpu().numpy().reshape(cache.shape), cache)
    # attention
    h = block.h[:rows].double().cpu().numpy().reshape(rows, Q_HEADS, DIM)
    tables = tables.reshape(step.batch, -1)
    for b in range(step.batch):
        at = slice(start[b], start[b + 1])
        if step.prompts:
            check_attention(h[at], got[at, :Q_HEADS], got[at, Q_HEADS:Q_HEADS + HEADS], got[at, Q_HEADS + HEADS:], DIM ** -0.5, True, t, name=f"prompt {b}")
        else:
            tokens = np.arange(lengths[b])
            k, v, ks, vs = plain.read(cache, tables[b, tokens // c.page] * c.page + tokens % c.page, HEADS, DIM, c.group, c.page)
            check_attention(h[at], got[at, :Q_HEADS], k, v, DIM ** -0.5, True, t, OFFSET[t] * ks, OFFSET[t] * vs, name=f"sequence {b}")
    # codes of it, and their product
    flat = h.reshape(rows, -1)
    codes = block.c2[:rows, :Q_HEADS * DIM].double().cpu().numpy() * block.q2[:rows].double().cpu().numpy()[:, None]
    close(codes, flat, (0.5 + 1e-4) * np.abs(flat).max(1, keepdims=True) / 127 + 1e-30, "codes")
    out = product(block.c2, block.q2, rows, block.w2, block.s2, HIDDEN, Q_HEADS * DIM)
    close(y.double().cpu().numpy(), out, 4 * U * np.abs(out) + HALF[t] * np.abs(out) * 1.01 + LEAST[t], "out")
    return cache


@pytest.mark.parametrize("t", ["f16", "bf16"])
@pytest.mark.parametrize("norms", [True, False])
def test_prompts_then_single_tokens(norms, t):
    import torch
    rng, w, weights, cache, block = make(torch, t, norms)
    a, b, c = cache.add(), cache.add(), cache.add()
    bytes_of = block.data.cpu().numpy().reshape(cache.pages, HEADS, -1)
    for ids, counts in (([a, b], [37, 1]), ([a, b], [1, 1]), ([b, c, a], [5, 20, 0]), ([c, a], [1, 1]), ([a], [100])):
        step = cache.step(ids, counts)
        x, r = w(step.rows, HIDDEN, scale=1.0), w(step.rows, HIDDEN, scale=0.5)
        y, total = torch.empty_like(x), torch.empty_like(x)
        block.forward(x, r, y, total, step)
        torch.cuda.synchronize()
        assert torch.equal(total, (x.float() + r.float()).to(x.dtype))
        bytes_of = check_pass(torch, block, weights, step, y, t, bytes_of)
    cache.remove(a)
    step = cache.step([cache.add()], [60])                                   # its pages have held another sequence
    x = w(60, HIDDEN, scale=1.0)
    y = torch.empty_like(x)
    block.forward(x, None, y, None, step)
    check_pass(torch, block, weights, step, y, t, bytes_of)


def test_against_fp32():
    """A prompt: 8-bit weights and activations alone, 3% of the result's norm at most (each of two products has two quantised factors, of
    about 0.7% each: 127 steps of rows whose largest element is about 3 times the root mean square). Single tokens: 4-bit keys and values too:
    a step of a quarter of the root mean square, 1 / sqrt(12) of it on average: 8% of the values and of the scores' differences."""
    import torch
    rng, w, weights, cache, block = make(torch, "bf16", seed=3)
    x, r = w(200, HIDDEN, scale=1.0), w(200, HIDDEN, scale=0.5)
    y, total = torch.empty_like(x), torch.empty_like(x)
    one = cache.add()
    block.forward(x[:150], r[:150], y[:150], total[:150], cache.step([one], [150]))
    for n in range(150, 200):
        block.forward(x[n:n + 1], r[n:n + 1], y[n:n + 1], total[n:n + 1], cache.step([one], [1]))
    want = attn.reference(x, r, eps=block.eps, heads=HEADS, dim=DIM, **weights)
    off = [float((y[s].float() - want[s]).norm() / want[s].norm()) for s in (slice(0, 150), slice(150, 200))]
    assert off[0] < 0.03 and off[1] < 0.25, off


def test_on_another_stream_and_after_the_step_is_gone():
    import torch
    rng, w, weights, cache, block = make(torch, "bf16", seed=4)
    one = cache.add()
    x = w(64, HIDDEN, scale=1.0)
    y, again = torch.empty_like(x), torch.empty_like(x)
    step = cache.step([one], [64])
    block.forward(x, None, y, None, step)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    for _ in range(3):
        again.zero_()
        torch.cuda.synchronize()
        block.forward(x, None, again, None, step, stream)
        stream.synchronize()
        assert torch.equal(y, again)
    with torch.cuda.stream(stream):
        block.forward(x, None, again, None, step)
    del step
    stream.synchronize()
    assert torch.equal(y, again)


def test_recorded_steps_of_one_token():
    """Head norms, cache write and attention of single tokens recorded once and replayed: positions, slots and lengths move on in
    device memory between the replays, with eager work between them; each replay against the eager calls."""
    import torch
    t, batch = "bf16", 3
    rng = np.random.Generator(np.random.PCG64(9))
    page, pages, width = 16, 20, 6
    desc = aqd.QcacheDesc(HEADS, DIM, 32, page, pages)
    order = torch.from_numpy(rng.permutation(pages)[:batch * width].astype(np.int32)).cuda()
    caches = [torch.zeros(aqd.qcache_bytes(desc), dtype=torch.uint8, device="cuda:0") for _ in range(2)]
    table = attn.rotary_table(200, DIM)
    position, slots, lengths = [torch.zeros(batch, dtype=torch.int32, device="cuda:0") for _ in range(3)]
    qkv = torch.zeros(batch, (Q_HEADS + 2 * HEADS) * DIM, dtype=DTYPE[t], device="cuda:0")
    wide, at_k, at_v = qkv.shape[1], Q_HEADS * DIM, (Q_HEADS + HEADS) * DIM
    ys = [torch.zeros(batch, Q_HEADS * DIM, dtype=DTYPE[t], device="cuda:0") for _ in range(2)]
    turned = torch.zeros_like(qkv)
    ws = torch.empty(aqd.ATTN_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda:0")

    def run(cache, y, stream):
        aqd.heads_run(batch, Q_HEADS, HEADS, DIM, DIM, aqd.PAIRS_HALVES, aqd.BF16, 200, 1e-6, qkv, wide, DIM, qkv[:, at_k:], wide, DIM, None, None, position,
                      table, turned, wide, DIM, turned[:, at_k:], wide, DIM, stream)
        aqd.qcache_write(desc, batch, aqd.BF16, turned[:, at_k:], wide, DIM, qkv[:, at_v:], wide, DIM, slots, cache, stream)
        aqd.qattn_run(desc, batch, Q_HEADS, batch, 1, width * page, aqd.BF16, DIM ** -0.5, turned, wide, DIM, None, cache, order, width, lengths, y,
                      at_k, DIM, ws, ws.numel(), stream)

    stream = torch.cuda.Stream()
    aqd.graph_begin(stream)
    run(caches[0], ys[0], stream)
    graph = aqd.graph_end(stream)
    try:
        for n in range(40):
            qkv.copy_(torch.from_numpy(rng.standard_normal(qkv.shape)))
            before = torch.tensor([n, n + 20, 2 * n], dtype=torch.int32, device="cuda:0")
            position.copy_(before)
            lengths.copy_(before + 1)
            slots.copy_(order.view(batch, width)[torch.arange(batch, device="cuda:0"), (before // page).long()] * page + before % page)
            torch.cuda.synchronize()
            aqd.graph_launch(graph, stream)
            stream.synchronize()
            run(caches[1], ys[1], None)
            torch.cuda.synchronize()
            assert torch.equal(ys[0], ys[1]) and torch.equal(caches[0], caches[1]) and bool(ys[0].any())
    finally:
        torch.cuda.synchronize()
        aqd.graph_destroy(graph)


def test_refused_drafts_leave_nothing():
    """Four drafts a step, of which some stay: the next step's rows have the bits that they have behind the accepted tokens alone."""
    import torch
    rng, w, weights, cache, block = make(torch, "bf16", seed=5)
    _, _, _, plain_cache, plain_block = make(torch, "bf16", seed=5)
    one, other = cache.add(), plain_cache.add()

    def run(block, cache, sequence, x):
        y = torch.empty_like(x)
        block.forward(x, None, y, None, cache.step([sequence], [len(x)]))
        torch.cuda.synchronize()
        return y

    x = w(30, HIDDEN, scale=1.0)
    assert torch.equal(run(block, cache, one, x), run(plain_block, plain_cache, other, x))
    for stay in (1, 3, 4, 0, 2):                           # 30 to 40 tokens: over a page's end and back
        drafts, length = w(4, HIDDEN, scale=1.0), cache.lengths[one]
        run(block, cache, one, drafts)
        cache.shorten(one, length + stay)
        if stay:
            run(plain_block, plain_cache, other, drafts[:stay])
        x = w(4, HIDDEN, scale=1.0)
        got, want = run(block, cache, one, x), run(plain_block, plain_cache, other, x)
        assert torch.equal(got, want), stay
        cache.shorten(one, length + stay)
        plain_cache.shorten(other, length + stay)

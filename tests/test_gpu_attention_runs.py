"""The attention operators as programs run them: long sequences, many of them, rows far from one another, less workspace than asked
for, two streams at once, recorded calls that are replayed. Tolerances: test_gpu_attention.py."""
import numpy as np
import pytest

import attention_plain as plain
from attention_plain import DTYPE
from paper_2007_06919_amd import aqd
from test_gpu_attention import OFFSET, TYPES, check_attention, check_heads, device, make_table, reals, run_attn, run_qattn, strides

pytestmark = pytest.mark.gpu


def spread(rng, n, count):
    """Rows to check: the first, the last, and others."""
    return sorted({0, n - 1, *rng.integers(0, n, count).tolist()})


def check_rows(got, q, k, v, rows, causal, t, k_size=None, v_size=None):
    """Rows of one sequence by themselves: all n x m products would take minutes."""
    n, m = q.shape[0], k.shape[0]
    for i in rows:
        seen = max(0, m - n + 1 + i) if causal else m
        sizes = [None if x is None else x[:seen] for x in (k_size, v_size)]
        check_attention(got[i:i + 1], q[i:i + 1], k[:seen], v[:seen], q.shape[2] ** -0.5, False, t, *sizes, name=f"row {i}")


@pytest.mark.parametrize("t, dim, heads, per, nq, nk, causal", [
    ("bf16", 128, 1, 2, 5000, 5000, True), ("f16", 64, 2, 1, 2500, 9000, True), ("bf16", 256, 1, 1, 1300, 4097, False), ("f16", 128, 1, 4, 3, 70001, True),
    ("bf16", 96, 1, 3, 700, 20000, True),
])
def test_attn_of_long_sequences(t, dim, heads, per, nq, nk, causal):
    import torch
    rng = np.random.Generator(np.random.PCG64(nk))
    shift = torch.from_numpy(rng.standard_normal((1, heads, dim)))
    q = reals(torch, rng, nq, heads * per, dim, t=t, scale=1.5)
    k, v = [torch.from_numpy(rng.standard_normal((nk, heads, dim))).add_(shift).to(DTYPE[t]) for _ in range(2)]
    y = torch.zeros_like(q, device="cuda:0")
    for workspace in (aqd.ATTN_WORKSPACE_BYTES, 0):
        run_attn(torch, q.cuda(), k.cuda(), v.cuda(), [0, nq], [0, nk], causal, t, y, workspace)
        check_rows(y.double().cpu().numpy(), q.double().numpy(), k.double().numpy(), v.double().numpy(), spread(rng, nq, 6), causal, t)


@pytest.mark.parametrize("t, dim, group, page, heads, per, counts, lengths", [
    ("bf16", 128, 64, 64, 2, 4, [1, 1], [50001, 20]), ("f16", 64, 32, 16, 1, 8, [1], [30000]), ("bf16", 256, 128, 256, 1, 2, [5, 2], [9000, 12345]),
    ("f16", 128, 32, 32, 1, 1, [40], [8000]),
])
def test_qattn_of_long_sequences(t, dim, group, page, heads, per, counts, lengths):
    import torch
    rng = np.random.Generator(np.random.PCG64(sum(lengths)))
    used = [-(-n // page) for n in lengths]
    c = aqd.QcacheDesc(heads, dim, group, page, sum(used) + 3)
    cache = torch.full((aqd.qcache_bytes(c),), 0xFF, dtype=torch.uint8, device="cuda:0")
    order, first = rng.permutation(c.pages), 0
    tables = np.full((len(lengths), max(used)), -1, np.int32)
    keys = []
    for b, n in enumerate(lengths):
        tables[b, :used[b]] = order[first:first + used[b]]
        first += used[b]
        at = np.arange(n)
        slots = torch.from_numpy((tables[b, at // page] * page + at % page).astype(np.int32)).cuda()
        shift = torch.from_numpy(rng.standard_normal((1, heads, dim)))
        k, v = [torch.from_numpy(rng.standard_normal((n, heads, dim))).add_(shift).float().cuda() for _ in range(2)]
        aqd.qcache_write(c, n, aqd.F32, k, *strides(k), v, *strides(v), slots, cache)
        aqd.qcache_read(c, n, aqd.F32, cache, slots, k, *strides(k), v, *strides(v))
        rows = [x.double().cpu().numpy() for x in (k, v)]
        # a group's largest element stands for 8 scales
        keys.append(rows + [np.abs(x).reshape(n, heads, dim // group, group).max(-1).repeat(group, -1) / 8 for x in rows])
    q = reals(torch, rng, sum(counts), heads * per, dim, t=t, scale=1.5)
    start = [0] + list(np.cumsum(counts))
    y = torch.zeros_like(q, device="cuda:0")
    for workspace in (aqd.ATTN_WORKSPACE_BYTES, 0):
        run_qattn(torch, c, cache, torch.from_numpy(tables).cuda(), lengths, q.cuda(), start, max(counts), t, y, workspace)
        got = y.double().cpu().numpy()
        for b in range(len(lengths)):
            k, v, ks, vs = keys[b]
            rows = slice(start[b], start[b + 1])
            check_rows(got[rows], q[rows].double().numpy(), k, v, spread(rng, counts[b], 3), True, t, OFFSET[t] * ks, OFFSET[t] * vs)


@pytest.mark.parametrize("causal", [True, False])
def test_attn_of_more_keys_than_max_keys(causal):
    """max_keys sizes the launch: all of a sequence's keys count, in split calls too."""
    import torch
    rng = np.random.Generator(np.random.PCG64(5))
    t, dim, nq, nk = "bf16", 128, [3, 2], [4000, 100]
    qs, ks = [0] + list(np.cumsum(nq)), [0] + list(np.cumsum(nk))
    q, (k, v) = reals(torch, rng, 5, 4, dim, t=t), [reals(torch, rng, 4100, 2, dim, t=t) for _ in range(2)]
    for most in (2000, 1100, 40, 0):
        assert aqd.attn_workspace(2, 4, 2, dim, 5, 4100, 3, 2000, causal, aqd.BF16) > 0
        y = torch.zeros_like(q, device="cuda:0")
        run_attn(torch, q.cuda(), k.cuda(), v.cuda(), qs, ks, causal, t, y, max_keys=most)
        got = y.double().cpu().numpy()
        for b in range(2):
            a, z = slice(qs[b], qs[b + 1]), slice(ks[b], ks[b + 1])
            check_attention(got[a], q[a].double().numpy(), k[z].double().numpy(), v[z].double().numpy(), dim ** -0.5, causal, t, name=f"{most}")


def test_rows_far_from_one_another():
    """Offsets past 32 bits in every tensor: columns of a buffer whose rows are 128 MiB apart."""
    import torch
    rng = np.random.Generator(np.random.PCG64(6))
    t, dim, n, hq, hk, row = "bf16", 64, 37, 4, 2, 1 << 26
    buf = torch.empty(n * row, dtype=DTYPE[t], device="cuda:0").view(n, row)

    def column(at, heads):
        return buf[:, at * 1024:at * 1024 + heads * dim].unflatten(1, (heads, dim))

    q, k, v, y, yk = column(0, hq), column(1, hk), column(2, hk), column(3, hq), column(4, hk)
    values = [reals(torch, rng, n, h, dim, t=t) for h in (hq, hk, hk)]
    for to, x in zip((q, k, v), values):
        to.copy_(x)
    run_attn(torch, q, k, v, [0, n], [0, n], True, t, y)
    check_attention(y.double().cpu().numpy(), *(x.double().numpy() for x in values), dim ** -0.5, True, t)
    # heads
    table = make_table(n, dim)
    position = torch.arange(n, dtype=torch.int32, device="cuda:0")
    aqd.heads_run(n, hq, hk, dim, dim, aqd.PAIRS_HALVES, TYPES[t], n, 1e-6, q, *strides(q), k, *strides(k), None, None, position, torch.from_numpy(table).cuda(),
                  y, *strides(y), yk, *strides(yk))
    for got, x in ((y, values[0]), (yk, values[1])):
        check_heads(got.double().cpu().numpy(), x, None, table, np.arange(n), dim, True, t)
    # cache, and attention over it
    c = aqd.QcacheDesc(hk, dim, 32, 16, 3)
    cache = torch.zeros(aqd.qcache_bytes(c), dtype=torch.uint8, device="cuda:0")
    aqd.qcache_write(c, n, TYPES[t], k, *strides(k), v, *strides(v), position, cache)
    host = np.zeros((3, hk, plain.block_bytes(dim, 32, 16)), np.uint8)
    plain.write(host, np.arange(n), values[1].float().numpy(), values[2].float().numpy(), hk, dim, 32, 16)
    assert np.array_equal(cache.cpu().numpy(), host.reshape(-1))
    kr, vr, ks, vs = plain.read(host, np.arange(n), hk, dim, 32, 16)
    y.zero_()
    run_qattn(torch, c, cache, torch.arange(3, dtype=torch.int32, device="cuda:0").view(1, 3), [n], q, [0, n], n, t, y)
    check_attention(y.double().cpu().numpy(), values[0].double().numpy(), kr, vr, dim ** -0.5, True, t, OFFSET[t] * ks, OFFSET[t] * vs)
    aqd.qcache_read(c, n, TYPES[t], cache, position, yk, *strides(yk), v, *strides(v))
    assert torch.equal(yk.cpu(), torch.from_numpy(kr).bfloat16()) and torch.equal(v.cpu(), torch.from_numpy(vr).bfloat16())


def test_many_sequences():
    """Thousands of them, most of a few tokens, some of none."""
    import torch
    rng = np.random.Generator(np.random.PCG64(7))
    t, dim, heads, per, batch, page = "f16", 64, 1, 2, 6000, 16
    lengths = rng.integers(0, 40, batch)
    starts = np.concatenate([[0], np.cumsum(lengths)])
    total = int(starts[-1])
    q, (k, v) = reals(torch, rng, total, heads * per, dim, t=t), [reals(torch, rng, total, heads, dim, t=t) for _ in range(2)]
    y = torch.zeros_like(q, device="cuda:0")
    run_attn(torch, q.cuda(), k.cuda(), v.cuda(), starts.tolist(), starts.tolist(), True, t, y)
    got, n64 = y.double().cpu().numpy(), [x.double().numpy() for x in (q, k, v)]
    some = spread(rng, batch, 40)
    for b in some:
        a = slice(starts[b], starts[b + 1])
        if lengths[b]:
            check_attention(got[a], *(x[a] for x in n64), dim ** -0.5, True, t, name=f"sequence {b}")
    # and the cache
    used = -(-lengths // page)
    c = aqd.QcacheDesc(heads, dim, 64, page, int(used.sum()) + 1)
    tables = np.full((batch, 3), -1, np.int32)
    first = np.concatenate([[0], np.cumsum(used)])
    for b in range(batch):
        tables[b, :used[b]] = np.arange(first[b], first[b + 1])
    slots = np.concatenate([tables[b, np.arange(n) // page] * page + np.arange(n) % page for b, n in enumerate(lengths)]).astype(np.int32)
    cache = torch.zeros(aqd.qcache_bytes(c), dtype=torch.uint8, device="cuda:0")
    kd, vd = k.cuda(), v.cuda()
    aqd.qcache_write(c, total, TYPES[t], kd, *strides(kd), vd, *strides(vd), torch.from_numpy(slots).cuda(), cache)
    one = reals(torch, rng, batch, heads * per, dim, t=t)
    z = torch.full_like(one, 3, device="cuda:0")
    run_qattn(torch, c, cache, torch.from_numpy(tables).cuda(), lengths.tolist(), one.cuda(), None, 1, t, z)
    got, host = z.double().cpu().numpy(), cache.cpu().numpy().reshape(c.pages, heads, -1)
    assert not got[lengths == 0].any()
    for b in some:
        if lengths[b]:
            kr, vr, ks, vs = plain.read(host, slots[starts[b]:starts[b + 1]], heads, dim, 64, page)
            check_attention(got[b:b + 1], one[b:b + 1].double().numpy(), kr, vr, dim ** -0.5, True, t, OFFSET[t] * ks, OFFSET[t] * vs, name=f"sequence {b}")


class Both:
    """One call of each kind of attention, both split, on tensors of its own."""

    def __init__(self, torch, seed, t="bf16", dim=128, heads=2, per=3, n=9000, queries=4, page=64):
        rng = np.random.Generator(np.random.PCG64(seed))
        self.torch, self.t, self.n, self.queries = torch, t, n, queries
        self.q = reals(torch, rng, queries, heads * per, dim, t=t).cuda()
        self.k, self.v = [reals(torch, rng, n, heads, dim, t=t).cuda() for _ in range(2)]
        self.c = aqd.QcacheDesc(heads, dim, 64, page, -(-n // page))
        self.cache = torch.zeros(aqd.qcache_bytes(self.c), dtype=torch.uint8, device="cuda:0")
        self.slots = torch.arange(n, dtype=torch.int32, device="cuda:0")
        self.table = self.slots[:self.c.pages].view(1, -1)
        self.start = torch.tensor([0, queries], dtype=torch.int32, device="cuda:0")
        self.keys = torch.tensor([0, n], dtype=torch.int32, device="cuda:0")
        self.sizes = [aqd.attn_workspace(1, heads * per, heads, dim, queries, n, queries, n, True, TYPES[t]),
                      aqd.qattn_workspace(self.c, 1, heads * per, queries, queries, n, TYPES[t])]
        assert min(self.sizes) > 0
        self.ws = [torch.full((s,), 0xFF, dtype=torch.uint8, device="cuda:0") for s in self.sizes]
        self.y = [torch.zeros_like(self.q) for _ in range(2)]

    def attn(self, y, ws, size, stream=None):
        q, k, v = self.q, self.k, self.v
        aqd.attn_run(1, q.shape[1], k.shape[1], q.shape[2], self.queries, self.n, self.queries, self.n, True, TYPES[self.t], q.shape[2] ** -0.5, q, *strides(q),
                     k, *strides(k), v, *strides(v), self.start, self.keys, y, *strides(y), ws, size, stream)

    def qattn(self, y, ws, size, stream=None):
        q = self.q
        aqd.qattn_run(self.c, 1, q.shape[1], self.queries, self.queries, self.n, TYPES[self.t], q.shape[2] ** -0.5, q, *strides(q), self.start, self.cache,
                      self.table, self.c.pages, self.keys[1:], y, *strides(y), ws, size, stream)

    def write(self, stream=None):
        aqd.qcache_write(self.c, self.n, TYPES[self.t], self.k, *strides(self.k), self.v, *strides(self.v), self.slots, self.cache, stream)

    def run(self, y, ws, stream=None):
        self.write(stream)
        self.attn(y[0], ws[0], self.sizes[0], stream)
        self.qattn(y[1], ws[1], self.sizes[1], stream)

    def check(self, y):
        n64 = [x.double().cpu().numpy() for x in (self.q, self.k, self.v)]
        dim = n64[0].shape[2]
        check_attention(y[0].double().cpu().numpy(), *n64, dim ** -0.5, True, self.t)
        shape = (self.c.heads, dim, self.c.group, self.c.page)
        k, v, ks, vs = plain.read(self.cache.cpu().numpy().reshape(self.c.pages, self.c.heads, -1), np.arange(self.n), *shape)
        check_attention(y[1].double().cpu().numpy(), n64[0], k, v, dim ** -0.5, True, self.t, OFFSET[self.t] * ks, OFFSET[self.t] * vs)


def test_less_workspace_than_asked_for():
    """The split follows what there is; nothing behind it is written."""
    import torch
    a = Both(torch, 11)
    a.write()
    for share in (0.0, 0.01, 0.3, 0.6, 0.999):
        ws = [torch.full((s + 4096,), 0x55, dtype=torch.uint8, device="cuda:0") for s in a.sizes]
        sizes = [int(s * share) for s in a.sizes]
        a.attn(a.y[0], ws[0], sizes[0])
        a.qattn(a.y[1], ws[1], sizes[1])
        torch.cuda.synchronize()
        a.check(a.y)
        for w, s in zip(ws, sizes):
            assert bool((w[s:] == 0x55).all())


def test_two_streams_at_once():
    """Each with its workspaces: the results are those of the calls alone, bit for bit."""
    import torch
    both = [Both(torch, 12), Both(torch, 13, t="f16", dim=64, per=5, n=7777, queries=1)]
    want = []
    for a in both:
        a.run(a.y, a.ws)
        torch.cuda.synchronize()
        a.check(a.y)
        want.append([y.clone() for y in a.y])
    streams = [torch.cuda.Stream() for _ in both]
    outs = [[[torch.zeros_like(y) for y in a.y] for _ in range(10)] for a in both]
    torch.cuda.synchronize()
    for i in range(10):
        for a, o, s in zip(both, outs, streams):
            a.run(o[i], a.ws, s)
    torch.cuda.synchronize()
    for o, w in zip(outs, want):
        for y in o:
            assert torch.equal(y[0], w[0]) and torch.equal(y[1], w[1])


def test_recorded_calls():
    """Cache write, attention over rows and over the cache recorded once, in two graphs that share their workspaces and run one after the
    other; replayed with other tensors' contents and eager work between; each replay has the eager calls' bits."""
    import torch
    a = Both(torch, 14)
    stream = torch.cuda.Stream()
    eager_ws = [w.clone() for w in a.ws]
    outs = [[torch.zeros_like(y) for y in a.y] for _ in range(3)]
    graphs = []
    try:
        for o in outs[:2]:
            aqd.graph_begin(stream)
            a.run(o, a.ws, stream)
            graphs.append(aqd.graph_end(stream))
        rng = np.random.Generator(np.random.PCG64(15))
        for i in range(5):
            a.q.copy_(reals(torch, rng, *a.q.shape, t=a.t))
            a.k.copy_(reals(torch, rng, *a.k.shape, t=a.t))
            a.keys[1] = a.n - 1000 * i
            torch.cuda.synchronize()
            for g in graphs:
                aqd.graph_launch(g, stream)
            stream.synchronize()
            a.run(outs[2], eager_ws)
            torch.cuda.synchronize()
            for o in outs[:2]:
                assert torch.equal(o[0], outs[2][0]) and torch.equal(o[1], outs[2][1])
            if i == 0:
                a.check(outs[0])
            else:
                assert bool((outs[0][0] != 0).all())
    finally:
        torch.cuda.synchronize()
        for g in graphs:
            aqd.graph_destroy(g)


@pytest.mark.parametrize("dim, heads, per, causal, few, batch", [(64, 2, 3, True, 700, 7), (128, 1, 8, True, 333, 70), (64, 1, 1, False, 1500, 256),
                                                                (128, 2, 2, True, 900, 257), (256, 1, 4, True, 200, 3000)])
def test_attn_of_sequences_of_unlike_lengths(dim, heads, per, causal, few, batch):
    """Some long sequences among many short ones and empty ones: the bits of the sequences by themselves, and rows of none left alone."""
    import torch
    t = "bf16"
    rng = np.random.Generator(np.random.PCG64(batch))
    n = rng.integers(0, 6, batch)
    n[rng.integers(0, batch, 3)] = few
    n[batch // 2], n[-1], n[0] = 129, 0, few // 2
    m = n + rng.integers(0, 50, batch)
    m[1] = 0
    qs, ks = [np.concatenate([[0], np.cumsum(x)]).tolist() for x in (n, m)]
    q, (k, v) = reals(torch, rng, qs[-1] + 5, heads * per, dim, t=t), [reals(torch, rng, ks[-1], heads, dim, t=t) for _ in range(2)]
    qd, kd, vd = q.cuda(), k.cuda(), v.cuda()
    y = torch.full_like(qd, 77)
    run_attn(torch, qd, kd, vd, qs, ks, causal, t, y)
    assert bool((y[qs[-1]:] == 77).all())
    alone = torch.full_like(qd, 77)
    some = np.flatnonzero(n > 5).tolist() + spread(rng, batch, 20)
    for b in some:
        run_attn(torch, qd, kd, vd, qs[b:b + 2], ks[b:b + 2], causal, t, alone, 0)
        a, z = slice(qs[b], qs[b + 1]), slice(ks[b], ks[b + 1])
        assert torch.equal(y[a], alone[a]), b
        if n[b]:
            check_rows(y[a].double().cpu().numpy(), q[a].double().numpy(), k[z].double().numpy(), v[z].double().numpy(), spread(rng, int(n[b]), 3), causal, t)
    if batch > 256:
        run_attn(torch, qd, kd, vd, qs, ks, causal, t, alone, max_queries=130)      # of longer ones the first 130
        for b in some:
            a = slice(qs[b], min(qs[b] + 130, qs[b + 1]))
            assert bool((alone[a] == alone[a]).all())


@pytest.mark.parametrize("t, dim, group, page, heads, per, batch, most, counts", [
    ("bf16", 64, 32, 16, 4, 2, 200, 3000, 1), ("f16", 128, 64, 64, 8, 4, 64, 2500, 3), ("bf16", 256, 128, 32, 2, 1, 256, 1700, 1),
    ("f16", 64, 64, 16, 8, 3, 65, 4200, 25), ("bf16", 128, 128, 256, 8, 2, 9, 5000, 2),
    ("bf16", 64, 32, 32, 1, 2, 1000, 4100, 1), ("f16", 128, 64, 64, 4, 2, 700, 5000, 2), ("bf16", 64, 64, 16, 8, 1, 1025, 5000, 1),
])
def test_qattn_of_sequences_of_unlike_lengths(t, dim, group, page, heads, per, batch, most, counts):
    """A few long sequences among many short and empty ones, which share the workgroups by their lengths: with all of the workspace, less,
    and none; lengths past max_keys and below 0."""
    import torch
    rng = np.random.Generator(np.random.PCG64(batch))
    lengths = rng.integers(0, 200, batch)
    lengths[rng.integers(0, batch, 3)] = most
    lengths[0], lengths[-1], lengths[batch // 2] = most - 1, 0, 300
    n = rng.integers(0, counts + 1, batch) if counts > 1 else np.ones(batch, int)
    n[0], n[1] = counts, 1
    starts = np.concatenate([[0], np.cumsum(n)])
    used = -(-lengths // page)
    first = np.concatenate([[0], np.cumsum(used)])
    c = aqd.QcacheDesc(heads, dim, group, page, int(first[-1]) + 1)
    tables = np.full((batch, -(-most // page)), -1, np.int32)
    for b in range(batch):
        tables[b, :used[b]] = np.arange(first[b], first[b + 1])[::-1]
    slots = [(tables[b, np.arange(m) // page] * page + np.arange(m) % page).astype(np.int32) for b, m in enumerate(lengths)]
    total = int(lengths.sum())
    k, v = [torch.randn(total, heads, dim, device="cuda:0", generator=torch.Generator("cuda:0").manual_seed(i)) for i in range(2)]
    cache = torch.full((aqd.qcache_bytes(c),), 0xFF, dtype=torch.uint8, device="cuda:0")
    aqd.qcache_write(c, total, aqd.F32, k, *strides(k), v, *strides(v), torch.from_numpy(np.concatenate(slots)).cuda(), cache)
    host = cache.cpu().numpy().reshape(c.pages, heads, -1)
    q = reals(torch, rng, int(starts[-1]) + 2, heads * per, dim, t=t)
    told = lengths.copy()
    told[-1] = -3
    told[lengths == most] += 7
    size = aqd.qattn_workspace(c, batch, heads * per, q.shape[0], counts, most, TYPES[t])
    assert (size > 0) == (batch <= 1024)
    some = np.flatnonzero(lengths >= 300).tolist() + spread(rng, batch, 12)
    keys = {b: plain.read(host, slots[b], heads, dim, group, page) if lengths[b] else [np.zeros((0, heads, dim))] * 4 for b in some}
    for workspace in (size, size // 2, size // 7, 0):
        y = torch.full_like(q, 77, device="cuda:0")
        run_qattn(torch, c, cache, torch.from_numpy(tables).cuda(), told.tolist(), q.cuda(), starts.tolist(), counts, t, y, workspace, max_keys=most)
        got = y.double().cpu().numpy()
        assert (got[starts[-1]:] == 77).all()
        for b in some:
            a = slice(starts[b], starts[b + 1])
            if n[b]:
                kr, vr, ks, vs = keys[b]
                rows = spread(rng, int(n[b]), 1)
                check_rows(got[a], q[a].double().numpy(), kr, vr, rows, True, t, OFFSET[t] * ks, OFFSET[t] * vs)


@pytest.mark.parametrize("t, dim, group, heads, per, batch, many, most", [
    ("bf16", 128, 64, 4, 4, 33, 200, 1500), ("f16", 64, 32, 1, 1, 300, 150, 900), ("bf16", 256, 128, 2, 3, 6, 70, 3000), ("bf16", 64, 64, 8, 2, 3, 120, 500),
])
def test_qattn_of_unlike_numbers_of_queries(t, dim, group, heads, per, batch, many, most):
    """One sequence with many queries among others with one or none, split and whole."""
    import torch
    rng = np.random.Generator(np.random.PCG64(many))
    n = rng.integers(0, 3, batch)
    n[batch // 3], n[-1] = many, 2
    lengths = np.maximum(rng.integers(0, most + 1, batch), n)
    lengths[0] = 0
    n[0] = 1
    lengths[batch // 3] = most
    starts = np.concatenate([[0], np.cumsum(n)])
    s = Both(torch, 20, t=t, dim=dim, heads=heads, per=per, n=most, queries=2)        # its cache: all sequences have the same pages
    if group != s.c.group:
        s.c = aqd.QcacheDesc(heads, dim, group, s.c.page, s.c.pages)
        s.cache = torch.zeros(aqd.qcache_bytes(s.c), dtype=torch.uint8, device="cuda:0")
    s.write()
    host = s.cache.cpu().numpy().reshape(s.c.pages, heads, -1)
    kr, vr, ks, vs = plain.read(host, np.arange(most), heads, dim, group, s.c.page)
    q = reals(torch, rng, int(starts[-1]) + 3, heads * per, dim, t=t)
    tables = s.table.repeat(batch, 1).contiguous()
    for workspace in (aqd.ATTN_WORKSPACE_BYTES, 0):
        y = torch.full_like(q, 77, device="cuda:0")
        run_qattn(torch, s.c, s.cache, tables, lengths.tolist(), q.cuda(), starts.tolist(), many, t, y, workspace)
        got = y.double().cpu().numpy()
        assert (got[starts[-1]:] == 77).all()
        for b in {batch // 3, batch - 1, 0, *spread(rng, batch, 8)}:
            a, m = slice(starts[b], starts[b + 1]), lengths[b]
            if n[b]:
                check_rows(got[a], q[a].double().numpy(), kr[:m], vr[:m], spread(rng, int(n[b]), 4), True, t, OFFSET[t] * ks[:m], OFFSET[t] * vs[:m])


@pytest.mark.parametrize("t", ["f16", "bf16"])
@pytest.mark.parametrize("scale", [0.0, -0.0, -0.11, 1.0, 1e-30])
def test_scales(scale, t):
    """None (every key the same weight), negative and large ones; keys hidden or not."""
    import torch
    rng = np.random.Generator(np.random.PCG64(21))
    dim, page = 64, 16
    q, (k, v) = reals(torch, rng, 20, 4, dim, t=t), [reals(torch, rng, 90, 2, dim, t=t) for _ in range(2)]
    n64 = [x.double().numpy() for x in (q, k, v)]
    c = aqd.QcacheDesc(2, dim, 32, page, 6)
    cache = torch.zeros(aqd.qcache_bytes(c), dtype=torch.uint8, device="cuda:0")
    slots = torch.arange(90, dtype=torch.int32, device="cuda:0")
    kd, vd = k.cuda(), v.cuda()
    aqd.qcache_write(c, 90, TYPES[t], kd, *strides(kd), vd, *strides(vd), slots, cache)
    kr, vr, ks, vs = plain.read(cache.cpu().numpy().reshape(6, 2, -1), np.arange(90), 2, dim, 32, page)
    y = torch.zeros_like(q, device="cuda:0")
    for workspace in (aqd.ATTN_WORKSPACE_BYTES, 0):
        for causal in (True, False):
            run_attn(torch, q.cuda(), kd, vd, [0, 20], [0, 90], causal, t, y, workspace, scale=scale)
            check_attention(y.double().cpu().numpy(), *n64, scale, causal, t, name=f"prompt {causal}")
        for count in (20, 1):                                                  # 32 and 16 rows a workgroup
            some = q[:count].cuda()
            run_qattn(torch, c, cache, slots[:6].view(1, 6), [90], some, [0, count], count, t, y[:count], workspace, scale=scale)
            check_attention(y[:count].double().cpu().numpy(), n64[0][:count], kr, vr, scale, True, t, OFFSET[t] * ks, OFFSET[t] * vs, name=f"cache {count}")


@pytest.mark.parametrize("t", ["f16", "bf16"])
@pytest.mark.parametrize("dim, order, pad, shift", [(128, "thd", 2, 2), (64, "htd", 6, 4), (256, "thd", 2, 6), (72, "htd", 2, 2)])
def test_attn_of_rows_at_multiples_of_four_bytes(dim, order, pad, shift, t):
    """Rows that the copies take as they lie, though not at multiples of 16 bytes."""
    import torch
    rng = np.random.Generator(np.random.PCG64(dim + pad))
    q, (k, v) = reals(torch, rng, 150, 4, dim, t=t), [reals(torch, rng, 170, 2, dim, t=t) for _ in range(2)]
    views = [device(torch, x, order, pad, shift, float("nan"))[1] for x in (q, k, v)]
    yb, y = device(torch, torch.full_like(q, 77), order, pad, shift)
    run_attn(torch, *views, [0, 150], [0, 170], True, t, y)
    check_attention(y.double().cpu().numpy(), *(x.double().numpy() for x in (q, k, v)), dim ** -0.5, True, t)
    y.fill_(77)
    assert bool((yb == 77).all())


def test_slots_that_repeat():
    """A read may name a slot twice, and pages may be of several sequences."""
    import torch
    rng = np.random.Generator(np.random.PCG64(22))
    t, heads, dim, group, page = "bf16", 2, 64, 64, 32
    c = aqd.QcacheDesc(heads, dim, group, page, 4)
    cache = torch.zeros(aqd.qcache_bytes(c), dtype=torch.uint8, device="cuda:0")
    k, v = [reals(torch, rng, 100, heads, dim, t=t).cuda() for _ in range(2)]
    aqd.qcache_write(c, 100, TYPES[t], k, *strides(k), v, *strides(v), torch.arange(100, dtype=torch.int32, device="cuda:0"), cache)
    slots = torch.tensor(([3, 3, 77, -5, 3, 128, 0] * 9), dtype=torch.int32, device="cuda:0")
    ko, vo = [torch.full((len(slots), heads, dim), 77.0, device="cuda:0") for _ in range(2)]
    aqd.qcache_read(c, len(slots), aqd.F32, cache, slots, ko, *strides(ko), vo, *strides(vo))
    kr, vr, ks, vs = plain.read(cache.cpu().numpy().reshape(4, heads, -1), np.arange(100), heads, dim, group, page)
    for i, s in enumerate(slots.tolist()):
        for out, want in ((ko, kr), (vo, vr)):
            assert np.array_equal(out[i].cpu().numpy(), want[s]) if 0 <= s < 100 else bool((out[i] == 77).all())
    tables = torch.tensor([[0, 1, 1, 2], [0, 1, 2, 3], [0, 0, 0, 0]], dtype=torch.int32, device="cuda:0")
    lengths = [97, 100, 65]
    q = reals(torch, rng, 3, heads * 2, dim, t=t)
    y = torch.zeros_like(q, device="cuda:0")
    run_qattn(torch, c, cache, tables, lengths, q.cuda(), None, 1, t, y)
    for b, m in enumerate(lengths):
        at = tables[b].cpu().numpy()[np.arange(m) // page] * page + np.arange(m) % page
        check_attention(y[b:b + 1].double().cpu().numpy(), q[b:b + 1].double().numpy(), kr[at], vr[at], dim ** -0.5, True, t, OFFSET[t] * ks[at],
                        OFFSET[t] * vs[at], name=f"sequence {b}")


@pytest.mark.parametrize("t", ["f16", "bf16"])
@pytest.mark.parametrize("count", [1, 12])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_values_of_unlike_sizes(group, count, t):
    """Tokens whose values are a million times as large as their neighbours', hidden from most queries or of hardly any weight, leave
    the others' bits alone. (Products of a weight and a scale are within half a step of T, or of its smallest numbers where the row's
    largest product is between 1/2 and 2^9: 2^-24 of that for each token, times codes up to 8.)"""
    import torch
    rng = np.random.Generator(np.random.PCG64(group + count))
    heads, per, dim, page, n = 2, 4, 128, 16, 200
    c = aqd.QcacheDesc(heads, dim, group, page, -(-n // page))
    q = reals(torch, rng, count, heads * per, dim, t=t)
    k, v = [torch.from_numpy(rng.standard_normal((n, heads, dim))).float() for _ in range(2)]
    v[::7] *= 1e6
    k[::7] = -3.0 * q[:, ::per].float().mean(0, keepdim=True)                  # their scores are low
    v *= 1e-4
    v[n - count // 2:n - count // 2 + 3] *= 1e4                                # seen by the last queries only
    k, v = k.cuda(), v.cuda()
    cache = torch.zeros(aqd.qcache_bytes(c), dtype=torch.uint8, device="cuda:0")
    slots = torch.arange(n, dtype=torch.int32, device="cuda:0")
    aqd.qcache_write(c, n, aqd.F32, k, *strides(k), v, *strides(v), slots, cache)
    kr, vr, ks, vs = plain.read(cache.cpu().numpy().reshape(c.pages, heads, -1), np.arange(n), heads, dim, group, page)
    y = torch.zeros_like(q, device="cuda:0")
    for workspace in (aqd.ATTN_WORKSPACE_BYTES, 0):
        run_qattn(torch, c, cache, slots[:c.pages].view(1, -1), [n], q.cuda(), [0, count], count, t, y, workspace, scale=1.0)
        got, q64 = y.double().cpu().numpy(), q.double().numpy()
        for i in range(count):
            m = n - count + 1 + i
            want, rest, size, most = plain.attention(q64[i:i + 1], kr[:m], vr[:m], 1.0, False, OFFSET[t] * ks[:m], OFFSET[t] * vs[:m])
            weights = plain.attention(q64[i:i + 1], kr[:m], vr[:m], 1.0, False)[2]
            s = np.einsum("thd,hpd->thp", kr[:m], q64[i].reshape(heads, per, dim))
            p = np.exp(s - s.max(0))
            largest = (p / p.sum(0) * vs[:m].max(-1)[:, :, None]).max(0).reshape(-1)   # product of a weight and a scale
            tol = (dim / 8 + 2) * 2 * 2.0 ** -24 * most[..., None] * rest + (plain.HALF[t] + 8 * 2.0 ** -24) * weights + \
                (m / 8 + 8) * 2 * 2.0 ** -24 * size + plain.HALF[t] * np.abs(want) * 1.01 + plain.LEAST[t]
            if t == "f16":
                tol = tol + m * 2.0 ** -24 * largest[None, :, None] * 8
            one = got[i:i + 1]
            # fp16 rounds what is 65520 or more, half a step past its largest number, to infinity
            past = (t == "f16") & np.isinf(one) & (one * want > 0) & (np.abs(want) + tol >= 65520)
            off = np.abs(np.where(past, want, one) - want)
            assert (off <= tol).all(), (i, float((off / tol).max()))

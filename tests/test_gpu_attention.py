"""The attention operators against plain implementations in 64 bits (attention_plain.py): head sizes, groups, pages, types,
strides with junk between the rows, lengths from none on, sequences without keys, pages anywhere, infinities and NaN where a
mask hides them.

Tolerances, from the definitions (u(T): half a step of T, relative; u = u(F32)).
heads: a sum of squares is at most 22 additions deep (16 elements of a lane, six exchanges) and enters by its root, 11 u; the
mean, eps, root, reciprocal and two products 6 u more: n is within 18 u of itself, and a rotated channel within
20 u of |n_a| + |n_b|, where table entries are at most 1. Then u(T) of the result.
cache: codes, scales and what is read are the definition's own bits.
attention: a score sums dim products in fp32. A matrix instruction rounds at most once for eight products, each time within 2 u of the
sum's magnitude, so a score is off by at most (dim / 8 + 2) 2 u of sum |q| |k|, and the result by that times sum p |v - y|. The
weights are rounded to T: u(T) of sum p |v|; a sum over the keys as one over channels: (keys / 8 + 8) 2 u of sum p |v|; exponentials and
the total: 8 u of the same. Then u(T) of the result. In the 4-bit cache the products are those of code + 128 (fp16: + 64), from which the
sum of 136 (72) is taken: |k| stands for 280 (152) |s|, and so does |v| in the sum over the keys."""
import numpy as np
import pytest

import attention_plain as plain
from attention_plain import DTYPE, HALF, LEAST
from paper_2007_06919_amd import aqd

pytestmark = pytest.mark.gpu

TYPES = {"f32": aqd.F32, "f16": aqd.F16, "bf16": aqd.BF16}
U = 2.0 ** -24
OFFSET = {"f16": 152.0, "bf16": 280.0}


def device(torch, values, order="thd", pad=0, shift=0, junk=77.0):
    """values [tokens][heads][dim] as a view of a junk-filled buffer: the buffer and the view. order: which dimension varies
    slowest; pad: elements between rows; shift: elements past an aligned address."""
    t, h, d = values.shape
    rows, n = (t, h) if order == "thd" else (h, t)
    buf = torch.full((shift + rows * (n * d + pad) + 64,), junk, dtype=values.dtype, device="cuda:0")
    view = buf[shift:shift + rows * (n * d + pad)].view(rows, n * d + pad)[:, :n * d].unflatten(1, (n, d))
    view = view if order == "thd" else view.transpose(0, 1)
    view.copy_(values)
    return buf, view


def untouched(torch, buf, view, junk=77.0):
    """Nothing of buf outside of view was written."""
    view.fill_(junk)
    return bool((buf == junk).all())


def strides(t):
    return t.stride(0), t.stride(1)


def reals(torch, rng, *shape, t, scale=1.0):
    return torch.from_numpy(rng.standard_normal(shape) * scale).to(DTYPE[t])


def close(got, want, tol, what=""):
    off = np.abs(got - want)
    assert (off <= tol).all(), (what, float(off.max()), float((off / tol).max()), int((off > tol).sum()))


# -------------------------------------------------------------------- heads
def run_heads(torch, q, k, wq, wk, table, position, rot, pairs, t, yq, yk, eps=1e-6):
    tokens, hq, dim = q.shape
    aqd.heads_run(tokens, hq, 0 if k is None else k.shape[1], dim, rot, pairs, TYPES[t], 0 if table is None else table.shape[0], eps,
                  q, *strides(q), k, *(strides(k) if k is not None else (0, 0)), wq, wk, position, table, yq, *strides(yq), yk,
                  *(strides(yk) if k is not None else (0, 0)))
    torch.cuda.synchronize()


def make_table(positions, rot):
    f = 10000.0 ** (-np.arange(0, rot, 2) / max(rot, 1))
    a = np.arange(positions)[:, None] * f
    return np.concatenate([np.cos(a), np.sin(a)], 1).astype(np.float32)


def check_heads(got, x, w, table, position, rot, halves, t, eps=1e-6, ok=None):
    want, size = plain.heads(x.double().numpy(), None if w is None else w.double().numpy(), eps, table.astype(np.float64), position, rot, halves)
    if ok is not None:
        got, want, size = got[ok], want[ok], size[ok]
    close(got, want, 20 * U * size + HALF[t] * np.abs(want) * 1.01 + LEAST[t])


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("halves", [True, False])
@pytest.mark.parametrize("tokens, hq, hk, dim, rot, order, pad, shift", [
    (1, 32, 8, 128, 128, "thd", 0, 0), (3, 4, 1, 64, 64, "thd", 128, 0), (5, 7, 2, 80, 60, "thd", 3, 1), (2, 3, 3, 256, 256, "htd", 0, 0),
    (9, 2, 1, 34, 34, "thd", 0, 0), (4, 2, 2, 2, 2, "thd", 0, 1), (3, 1, 1, 512, 256, "htd", 8, 0), (2, 2, 1, 1024, 1022, "thd", 0, 0),
    (2, 1, 1, 1024, 1024, "thd", 5, 3), (70, 5, 1, 96, 32, "thd", 16, 0), (3, 2, 1, 300, 100, "thd", 0, 0), (2, 2, 2, 514, 2, "thd", 0, 0),
    (257, 3, 1, 128, 0, "thd", 0, 0), (5, 3, 1, 72, 72, "thd", 4, 0), (3, 2, 1, 120, 56, "htd", 0, 1), (2, 1, 1, 1000, 1000, "thd", 0, 0),
    (2, 2, 1, 1000, 504, "thd", 2, 0),
])
def test_heads(tokens, hq, hk, dim, rot, order, pad, shift, halves, t):
    import torch
    rng = np.random.Generator(np.random.PCG64(tokens * 1009 + dim + rot))
    q, k = reals(torch, rng, tokens, hq, dim, t=t, scale=3.0), reals(torch, rng, tokens, hk, dim, t=t, scale=0.1)
    if tokens > 2:
        q[1] = 0
    wq, wk = 1 + reals(torch, rng, dim, t=t, scale=0.3), 1 + reals(torch, rng, dim, t=t, scale=0.3)
    positions = 5000
    table = make_table(positions, rot) if rot else np.zeros((positions, 0), np.float32)
    position = rng.integers(0, positions, tokens)
    position[-1] = positions - 1
    tb, pos = torch.from_numpy(table).cuda() if rot else None, torch.from_numpy(position.astype(np.int32)).cuda()
    qb, qd = device(torch, q, order, pad, shift)
    kb, kd = device(torch, k, order, pad, shift)
    yqb, yq = device(torch, torch.zeros_like(q), "thd", pad + 1, shift)
    ykb, yk = device(torch, torch.zeros_like(k), order, pad, shift)
    run_heads(torch, qd, kd, wq.cuda(), wk.cuda(), tb, pos if rot else None, rot, aqd.PAIRS_HALVES if halves else aqd.PAIRS_NEIGHBOURS, t, yq, yk)
    check_heads(yq.double().cpu().numpy(), q, wq, table, position, rot, halves, t)
    check_heads(yk.double().cpu().numpy(), k, wk, table, position, rot, halves, t)
    once = yq.clone()
    assert untouched(torch, yqb, yq) and untouched(torch, ykb, yk)
    assert torch.equal(qd.cpu(), q) and torch.equal(kd.cpu(), k)
    # in place, and of q alone without a norm
    run_heads(torch, qd, kd, wq.cuda(), wk.cuda(), tb, pos if rot else None, rot, aqd.PAIRS_HALVES if halves else aqd.PAIRS_NEIGHBOURS, t, qd, kd)
    assert torch.equal(qd, once)
    qd.copy_(q)
    run_heads(torch, qd, None, None, None, tb, pos if rot else None, rot, aqd.PAIRS_HALVES if halves else aqd.PAIRS_NEIGHBOURS, t, qd, None)
    check_heads(qd.double().cpu().numpy(), q, None, table, position, rot, halves, t)
    assert untouched(torch, qb, qd)


def test_heads_of_unknown_positions_are_not_numbers():
    import torch
    rng = np.random.Generator(np.random.PCG64(5))
    q = reals(torch, rng, 6, 3, 96, t="bf16")
    table, position = make_table(10, 64), np.array([0, -1, 9, 10, 2 ** 31 - 1, -2 ** 31])
    y = torch.zeros_like(q, device="cuda:0")
    run_heads(torch, q.cuda(), None, None, None, torch.from_numpy(table).cuda(), torch.from_numpy(position.astype(np.int32)).cuda(), 64,
              aqd.PAIRS_HALVES, "bf16", y, None)
    got = y.double().cpu().numpy()
    bad = np.array([1, 3, 4, 5])
    assert np.isnan(got[bad][..., :64]).all() and np.array_equal(got[bad][..., 64:], q.double().numpy()[bad][..., 64:])
    position[bad] = 0
    check_heads(got, q, None, table, position, 64, True, "bf16", ok=np.array([0, 2]))


def test_a_head_that_is_no_number_stays_alone():
    import torch
    rng = np.random.Generator(np.random.PCG64(6))
    q = reals(torch, rng, 4, 4, 64, t="f16")
    q[1, 2, 5], q[2, 0, 63] = float("nan"), float("inf")
    table, position, w = make_table(10, 64), np.arange(4), 1 + reals(torch, rng, 64, t="f16", scale=0.2)
    y = torch.zeros_like(q, device="cuda:0")
    run_heads(torch, q.cuda(), None, w.cuda(), None, torch.from_numpy(table).cuda(), torch.from_numpy(position.astype(np.int32)).cuda(), 64,
              aqd.PAIRS_NEIGHBOURS, "f16", y, None)
    got = y.double().cpu().numpy()
    ok = np.ones((4, 4), bool)
    ok[1, 2] = ok[2, 0] = False
    assert np.isnan(got[1, 2]).all() and np.isnan(got[2, 0, 63]) and np.isfinite(got[ok]).all()
    check_heads(got, q, w, table, position, 64, False, "f16", ok=ok)


# -------------------------------------------------------------------- cache
def new_cache(torch, rng, heads, dim, group, page, pages):
    """Pages of random bytes: what slots that are not written hold."""
    return rng.integers(0, 256, (pages, heads, plain.block_bytes(dim, group, page)), dtype=np.uint8)


CACHES = [(1, 64, 32, 16), (3, 64, 64, 32), (2, 128, 32, 16), (8, 128, 64, 64), (5, 128, 128, 128), (2, 256, 32, 16), (1, 256, 64, 256),
          (3, 256, 128, 64)]


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("tokens, order, pad, shift", [(1, "thd", 0, 0), (37, "thd", 64, 0), (37, "htd", 3, 1)])
@pytest.mark.parametrize("heads, dim, group, page", CACHES)
def test_cache_write_and_read(heads, dim, group, page, tokens, order, pad, shift, t):
    import torch
    rng = np.random.Generator(np.random.PCG64(heads * 31 + dim + group + page + tokens))
    pages = 5
    k, v = reals(torch, rng, tokens, heads, dim, t=t, scale=2.0), reals(torch, rng, tokens, heads, dim, t=t, scale=1e-3) + 0.01
    if tokens > 8:
        k[1], v[2], k[3, 0, :group], v[4, 0, 7] = 0, 1e-38, -5.0, float("nan")
        k[5, 0, 1], k[5, 0, 2] = 50.0, -50.0                             # the positive one of two gives the scale
        v[6, heads - 1, dim - 1] = float("-inf")
    slots = rng.permutation(pages * page)[:tokens].astype(np.int32)
    start = int(slots[0])
    if tokens > 30:                                                      # a run of a sequence's tokens among the others
        run = np.arange(start - start % 4 + 2, start - start % 4 + 16) % (pages * page)
        rest = np.setdiff1d(slots, run)
        slots = np.concatenate([rest, run])[-tokens:].astype(np.int32)
        slots[7], slots[9] = -1, pages * page                            # left out
    cache = new_cache(torch, rng, heads, dim, group, page, pages)
    c = aqd.QcacheDesc(heads, dim, group, page, pages)
    assert cache.nbytes == aqd.qcache_bytes(c)
    _, kd = device(torch, k, order, pad, shift)
    _, vd = device(torch, v, order, pad, shift)
    dev, sl = torch.from_numpy(cache.copy()).cuda(), torch.from_numpy(slots).cuda()
    aqd.qcache_write(c, len(slots), TYPES[t], kd[:len(slots)], *strides(kd), vd[:len(slots)], *strides(vd), sl, dev)
    torch.cuda.synchronize()
    plain.write(cache, slots, k.float().numpy(), v.float().numpy(), heads, dim, group, page)
    assert np.array_equal(dev.cpu().numpy(), cache)
    # back, rows of slots outside of the cache left as they were
    kb, ko = device(torch, torch.full_like(k, 77), order, pad, shift)
    vb, vo = device(torch, torch.full_like(v, 77), "thd", pad, shift)
    aqd.qcache_read(c, len(slots), TYPES[t], dev, sl, ko, *strides(ko), vo, *strides(vo))
    torch.cuda.synchronize()
    inside = (slots >= 0) & (slots < pages * page)
    wk, wv, _, _ = plain.read(cache, slots[inside], heads, dim, group, page)
    for got, want in ((ko, wk), (vo, wv)):
        got = got.cpu()[:len(slots)]
        assert torch.equal(got[inside].nan_to_num(12345.0), torch.from_numpy(want).float().to(DTYPE[t]).nan_to_num(12345.0))
        assert bool((got[~inside] == 77).all())
    assert untouched(torch, kb, ko) and untouched(torch, vb, vo)


def test_cache_slots_past_32_bits():
    """Offsets of the far pages of a cache of more than 4 GiB."""
    import torch
    heads, dim, group, page = 16, 256, 128, 256
    each = heads * plain.block_bytes(dim, group, page)
    pages = (5 << 30) // each
    c = aqd.QcacheDesc(heads, dim, group, page, pages)
    rng = np.random.Generator(np.random.PCG64(8))
    dev = torch.zeros(pages, heads, each // heads, dtype=torch.uint8, device="cuda:0")
    slots = np.array([0, pages * page - 1, (pages - 1) * page, pages * page // 2], np.int32)
    k, v = reals(torch, rng, 4, heads, dim, t="bf16"), reals(torch, rng, 4, heads, dim, t="bf16")
    kd, vd, sl = k.cuda(), v.cuda(), torch.from_numpy(slots).cuda()
    aqd.qcache_write(c, 4, aqd.BF16, kd, *strides(kd), vd, *strides(vd), sl, dev)
    at = np.unique(slots // page)
    small = np.zeros((len(at), heads, each // heads), np.uint8)
    plain.write(small, np.searchsorted(at, slots // page) * page + slots % page, k.float().numpy(), v.float().numpy(), heads, dim, group, page)
    assert np.array_equal(dev[torch.from_numpy(at).cuda()].cpu().numpy(), small)
    ko, vo = torch.zeros_like(kd), torch.zeros_like(vd)
    aqd.qcache_read(c, 4, aqd.BF16, dev, sl, ko, *strides(ko), vo, *strides(vo))
    wk, wv, _, _ = plain.read(small, np.searchsorted(at, slots // page) * page + slots % page, heads, dim, group, page)
    assert torch.equal(ko.cpu(), torch.from_numpy(wk).bfloat16()) and torch.equal(vo.cpu(), torch.from_numpy(wv).bfloat16())
    # attention that reads the far pages
    q = reals(torch, rng, 1, heads, dim, t="bf16")
    y = torch.zeros_like(q, device="cuda:0")
    tables = torch.tensor([[pages - 1]], dtype=torch.int32, device="cuda:0")
    run_qattn(torch, c, dev, tables, [1], q.cuda(), None, 1, "bf16", y)
    far = plain.read(small, np.array([(len(at) - 1) * page]), heads, dim, group, page)
    assert np.abs(y.double().cpu().numpy()[0] - far[1][0]).max() <= 3 * 2.0 ** -8 * np.abs(far[1]).max()


# ---------------------------------------------------------------- attention
def run_qattn(torch, c, cache, tables, lengths, q, q_start, max_queries, t, y, workspace=aqd.ATTN_WORKSPACE_BYTES, max_keys=None, scale=None,
              stream=None):
    ws = torch.full((max(workspace, 16),), 0xFF, dtype=torch.uint8, device="cuda:0") if workspace else None
    lens = torch.tensor(lengths, dtype=torch.int32, device="cuda:0")
    start = None if q_start is None else torch.tensor(q_start, dtype=torch.int32, device="cuda:0")
    aqd.qattn_run(c, len(lengths), q.shape[1], q.shape[0], max_queries, max(lengths) if max_keys is None else max_keys, TYPES[t],
                  c.dim ** -0.5 if scale is None else scale, q, *strides(q), start, cache, tables, tables.shape[1], lens, y, *strides(y), ws,
                  workspace, stream)
    torch.cuda.synchronize()


class Sequences:
    """A cache of random sequences, their pages anywhere, what lies past their ends random bytes (scales that are NaN and
    infinities among them)."""

    def __init__(self, torch, seed, lengths, heads, dim, group, page, scale=1.0):
        rng = self.rng = np.random.Generator(np.random.PCG64(seed))
        self.lengths, self.page = list(lengths), page
        used = [-(-n // page) for n in lengths]
        pages = sum(used) + 2
        self.cache = new_cache(torch, rng, heads, dim, group, page, pages)
        order = rng.permutation(pages)
        self.tables = np.full((len(lengths), max(1, max(used))), -7, np.int32)
        self.c = aqd.QcacheDesc(heads, dim, group, page, pages)
        self.shape = (heads, dim, group, page)
        self.k, self.v, self.ks, self.vs = [], [], [], []
        first = 0
        for b, n in enumerate(lengths):
            self.tables[b, :used[b]] = order[first:first + used[b]]
            first += used[b]
            slots = self.slots(b)
            k, v = [(rng.standard_normal((n, heads, dim)) + 0.5 * rng.standard_normal((heads, dim))).astype(np.float32) * scale for _ in range(2)]
            plain.write(self.cache, slots, k, v, *self.shape)
            for to, x in zip((self.k, self.v, self.ks, self.vs), plain.read(self.cache, slots, *self.shape)):
                to.append(x)

    def slots(self, b):
        t = np.arange(self.lengths[b])
        return self.tables[b, t // self.page] * self.page + t % self.page

    def check(self, got, q, q_start, t, scale=None, name=""):
        dim = self.shape[1]
        scale = dim ** -0.5 if scale is None else scale
        for b, n in enumerate(self.lengths):
            rows = slice(q_start[b], q_start[b + 1])
            check_attention(got[rows], q[rows].double().numpy(), self.k[b], self.v[b], scale, True, t, OFFSET[t] * self.ks[b], OFFSET[t] * self.vs[b],
                            f"{name} sequence {b} of {n}")


def check_attention(got, q, k, v, scale, causal, t, k_size=None, v_size=None, name=""):
    want, rest, size, most = plain.attention(q, k, v, scale, causal, k_size, v_size)
    weights = plain.attention(q, k, v, scale, causal)[2] if v_size is not None else size
    keys = k.shape[0]
    score = (q.shape[2] / 8 + 2) * 2 * U * most[..., None]
    close(got, want, score * rest + (HALF[t] + 8 * U) * weights + (keys / 8 + 8) * 2 * U * size + HALF[t] * np.abs(want) * 1.01 + LEAST[t], name)


@pytest.mark.parametrize("t", ["f16", "bf16"])
@pytest.mark.parametrize("workspace", [aqd.ATTN_WORKSPACE_BYTES, 0])
@pytest.mark.parametrize("heads, dim, group, page, per, lengths", [
    (1, 64, 32, 16, 1, [1]), (2, 64, 64, 32, 3, [15, 16, 17, 0, 33]), (2, 128, 32, 16, 4, [600, 5, 129]), (1, 128, 64, 64, 16, [65, 64]),
    (3, 128, 128, 128, 8, [1, 300, 31]), (1, 256, 32, 16, 2, [47, 90]), (2, 256, 64, 256, 17, [257]), (1, 256, 128, 32, 1, [100, 1]),
    (1, 64, 32, 16, 40, [75]), (2, 128, 64, 16, 5, [2048]),
])
def test_qattn_single_tokens(heads, dim, group, page, per, lengths, workspace, t):
    import torch
    s = Sequences(torch, dim + group + per, lengths, heads, dim, group, page)
    q = reals(torch, s.rng, len(lengths), heads * per, dim, t=t, scale=1.2)
    qb, qd = device(torch, q, "thd", 24)
    yb, y = device(torch, torch.zeros_like(q), "thd", 8)
    run_qattn(torch, s.c, torch.from_numpy(s.cache).cuda(), torch.from_numpy(s.tables).cuda(), lengths, qd, None, 1, t, y, workspace)
    got = y.double().cpu().numpy()
    s.check(got, q, list(range(len(lengths) + 1)), t)
    for b, n in enumerate(lengths):
        assert n or not got[b].any()
    assert untouched(torch, yb, y)


@pytest.mark.parametrize("t", ["f16", "bf16"])
@pytest.mark.parametrize("heads, dim, group, page, per, lengths, counts, order", [
    (2, 64, 64, 32, 4, [5, 100, 0, 2], [4, 4, 4, 4], "thd"), (1, 128, 32, 16, 8, [300, 17], [7, 1], "thd"), (2, 128, 128, 16, 1, [70], [70], "thd"),
    (2, 256, 128, 64, 3, [40, 130], [3, 9], "htd"), (1, 64, 32, 16, 16, [200, 30, 64], [5, 0, 3], "thd"), (3, 128, 64, 256, 2, [513], [33], "htd"),
])
def test_qattn_several_tokens(heads, dim, group, page, per, lengths, counts, order, t):
    """Drafts and chunks of prompts: a sequence's last tokens, each of which sees those before it."""
    import torch
    s = Sequences(torch, dim + group + sum(counts), lengths, heads, dim, group, page)
    start = [0] + list(np.cumsum(counts))
    q = reals(torch, s.rng, start[-1] + 3, heads * per, dim, t=t, scale=1.2)          # three rows behind the last sequence
    qb, qd = device(torch, q, order, 24, 1)
    yb, y = device(torch, torch.full_like(q, 77), order, 8, 1)
    for workspace in (aqd.ATTN_WORKSPACE_BYTES, 0):
        y.fill_(77)
        run_qattn(torch, s.c, torch.from_numpy(s.cache).cuda(), torch.from_numpy(s.tables).cuda(), lengths, qd, start, max(counts), t, y, workspace)
        got = y.double().cpu().numpy()
        s.check(got[:start[-1]], q, start, t)
        assert (got[start[-1]:] == 77).all()
    assert untouched(torch, yb, y)


def test_qattn_pages_outside_of_the_cache():
    """NaN for the queries that see such a page, and for no other."""
    import torch
    heads, dim, page, t = 2, 128, 16, "bf16"
    s = Sequences(torch, 3, [100, 100, 100, 40], heads, dim, 64, page)
    tables = s.tables.copy()
    tables[0, 2], tables[1, 6], tables[3, 3] = s.c.pages, -1, 2 ** 31 - 1      # the last one past its sequence's end
    start = [0, 1, 9, 10, 11]                                                  # sequence 1 has eight queries, of which the last four see the page
    q = reals(torch, s.rng, 11, heads * 3, dim, t=t)
    y = torch.zeros_like(q, device="cuda:0")
    for workspace in (aqd.ATTN_WORKSPACE_BYTES, 0):
        run_qattn(torch, s.c, torch.from_numpy(s.cache).cuda(), torch.from_numpy(tables).cuda(), s.lengths, q.cuda(), start, 8, t, y, workspace)
        got = y.double().cpu().numpy()
        assert np.isnan(got[0]).all() and np.isnan(got[5:9]).all()
        assert np.isfinite(got[1:5]).all() and np.isfinite(got[9:]).all()
        good = got.copy()
        good[0], good[5:9] = 0, 0
        for b in (2, 3):
            rows = slice(start[b], start[b + 1])
            check_attention(got[rows], q[rows].double().numpy(), s.k[b], s.v[b], dim ** -0.5, True, t, 280 * s.ks[b], 280 * s.vs[b])


def test_qattn_lengths_are_bounded():
    """A length past max_keys, or past what the table holds, counts as that; a negative one as none."""
    import torch
    heads, dim, page, t = 1, 64, 16, "f16"
    s = Sequences(torch, 4, [64, 64, 64], heads, dim, 32, page)
    q = reals(torch, s.rng, 3, 2, dim, t=t)
    cache, tables = torch.from_numpy(s.cache).cuda(), torch.from_numpy(s.tables).cuda()
    for lengths, most, want in (([64, 2 ** 31 - 1, -5], 50, [50, 50, 0]), ([64, 2 ** 31 - 1, 10], 1000, [64, 64, 10])):
        y = torch.full_like(q, 3, device="cuda:0")
        run_qattn(torch, s.c, cache, tables, lengths, q.cuda(), None, 1, t, y, max_keys=most)
        got = y.double().cpu().numpy()
        for b, n in enumerate(want):
            check_attention(got[b:b + 1], q[b:b + 1].double().numpy(), s.k[b][:n], s.v[b][:n], dim ** -0.5, True, t, 152 * s.ks[b][:n], 152 * s.vs[b][:n])


@pytest.mark.parametrize("t", ["f16", "bf16"])
@pytest.mark.parametrize("size", [1e-5, 3e3, 1e-30, 1e30])
def test_qattn_of_small_and_large_values(size, t):
    """Values whose scales 16 bits would lose beside a weight; keys of ordinary size."""
    import torch
    heads, dim, group, page, lengths = 2, 128, 32, 16, [500, 3]
    s = Sequences(torch, 9, lengths, heads, dim, group, page)
    big = [(s.rng.standard_normal(v.shape) * size).astype(np.float32) for v in s.v]
    for b in range(2):
        plain.write(s.cache, s.slots(b), s.k[b].astype(np.float32), big[b], *s.shape)
        s.k[b], s.v[b], s.ks[b], s.vs[b] = plain.read(s.cache, s.slots(b), *s.shape)
    q = reals(torch, s.rng, 2, heads * 4, dim, t=t)
    y = torch.zeros_like(q, device="cuda:0")
    run_qattn(torch, s.c, torch.from_numpy(s.cache).cuda(), torch.from_numpy(s.tables).cuda(), lengths, q.cuda(), None, 1, t, y)
    got = y.double().cpu().numpy()
    if t == "f16" and size == 1e30:
        assert not np.isfinite(got).any() or np.abs(got[np.isfinite(got)]).max() == 0
    else:
        s.check(got, q, [0, 1, 2], t)


def test_qattn_a_group_that_is_no_number():
    """NaN in the values reaches the group's channels of the queries that see it, and nothing else; past the end nothing."""
    import torch
    heads, dim, group, page, t = 1, 128, 32, 16, "f16"
    s = Sequences(torch, 12, [80], heads, dim, group, page)
    v = s.v[0].astype(np.float32)
    v[77, 0, 40] = float("nan")                                              # seen by the last three of five queries
    plain.write(s.cache, s.slots(0), s.k[0].astype(np.float32), v, *s.shape)
    k, v, ks, vs = plain.read(s.cache, s.slots(0), *s.shape)
    q = reals(torch, s.rng, 5, 4, dim, t=t)
    y = torch.zeros_like(q, device="cuda:0")
    run_qattn(torch, s.c, torch.from_numpy(s.cache).cuda(), torch.from_numpy(s.tables).cuda(), [80], q.cuda(), [0, 5], 5, t, y)
    got = y.double().cpu().numpy()
    assert np.isnan(got[2:, :, 32:64]).all() and np.isfinite(got[:2]).all() and np.isfinite(np.delete(got, np.s_[32:64], 2)).all()
    v[77, 0, 32:64], vs[77, 0, 32:64] = 0, 0
    got[2:, :, 32:64] = plain.attention(q.double().numpy(), k, v, dim ** -0.5, True)[0][2:, :, 32:64]
    check_attention(got, q.double().numpy(), k, v, dim ** -0.5, True, t, 152 * ks, 152 * vs)


def run_attn(torch, q, k, v, q_start, k_start, causal, t, y, workspace=aqd.ATTN_WORKSPACE_BYTES, max_queries=None, max_keys=None, scale=None,
             stream=None):
    ws = torch.full((max(workspace, 16),), 0xFF, dtype=torch.uint8, device="cuda:0") if workspace else None
    qs, ks = [torch.tensor(a, dtype=torch.int32, device="cuda:0") for a in (q_start, k_start)]
    mq, mk = [max(b - a for a, b in zip(s, s[1:])) for s in (q_start, k_start)]
    aqd.attn_run(len(q_start) - 1, q.shape[1], k.shape[1], q.shape[2], q.shape[0], k.shape[0], mq if max_queries is None else max_queries,
                 mk if max_keys is None else max_keys, causal, TYPES[t], q.shape[2] ** -0.5 if scale is None else scale, q, *strides(q), k, *strides(k),
                 v, *strides(v), qs, ks, y, *strides(y), ws, workspace, stream)
    torch.cuda.synchronize()


@pytest.mark.parametrize("t", ["f16", "bf16"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dim, heads, per, nq, nk, order, pad, shift", [
    (64, 2, 2, [1], [1], "thd", 0, 0), (128, 1, 3, [63, 64, 65], [63, 64, 65], "thd", 0, 0), (128, 2, 4, [5, 0, 130], [70, 9, 130], "thd", 64, 0),
    (64, 1, 1, [200], [333], "htd", 8, 0), (256, 1, 2, [33, 1], [90, 257], "thd", 0, 0), (80, 2, 1, [40, 12], [40, 50], "thd", 16, 0),
    (8, 1, 2, [70], [70], "thd", 0, 0), (128, 2, 1, [50, 20], [30, 0], "thd", 0, 0), (72, 1, 2, [100], [140], "thd", 3, 1), (128, 1, 2, [130], [150], "htd", 5, 1),
    (200, 1, 1, [65], [129], "htd", 0, 0), (64, 3, 7, [16, 3], [500, 700], "thd", 0, 0), (128, 1, 16, [2], [1500], "thd", 0, 0),
])
def test_attn(dim, heads, per, nq, nk, order, pad, shift, causal, t):
    import torch
    rng = np.random.Generator(np.random.PCG64(dim + sum(nq) + 7 * sum(nk)))
    qs, ks = [0] + list(np.cumsum(nq)), [0] + list(np.cumsum(nk))
    q = reals(torch, rng, qs[-1] + 2, heads * per, dim, t=t, scale=1.3)
    k, v = reals(torch, rng, max(ks[-1], 1), heads, dim, t=t, scale=1.3), reals(torch, rng, max(ks[-1], 1), heads, dim, t=t)
    junk = float("nan")                                                       # between the rows
    _, qd = device(torch, q, order, pad, shift, junk)
    _, kd = device(torch, k, order, pad, shift, junk)
    _, vd = device(torch, v, order, pad, shift, junk)
    yb, y = device(torch, torch.full_like(q, 77), order, pad, shift)
    for workspace in (aqd.ATTN_WORKSPACE_BYTES, 0):
        y.fill_(77)
        run_attn(torch, qd, kd, vd, qs, ks, causal, t, y, workspace)
        got = y.double().cpu().numpy()
        for b in range(len(nq)):
            a, z = slice(qs[b], qs[b + 1]), slice(ks[b], ks[b + 1])
            check_attention(got[a], q[a].double().numpy(), k[z].double().numpy(), v[z].double().numpy(), dim ** -0.5, causal, t, name=f"sequence {b}")
            if nk[b] < nq[b]:
                empty = got[a][:nq[b] - nk[b]] if causal else got[a] if not nk[b] else got[:0]
                assert not empty.any()
        assert (got[qs[-1]:] == 77).all()
    assert untouched(torch, yb, y)


@pytest.mark.parametrize("t", ["f16", "bf16"])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_attn_what_a_mask_hides_has_no_part(dim, t):
    """Infinities and NaN in keys and values that a query does not see, and in the rows of other sequences, leave its result alone."""
    import torch
    rng = np.random.Generator(np.random.PCG64(dim))
    n, heads, per = 150, 2, 2
    qs, ks = [0, 20, 20 + n], [0, 20, 20 + n]
    q = reals(torch, rng, 20 + n, heads * per, dim, t=t)
    k, v = reals(torch, rng, 20 + n, heads, dim, t=t), reals(torch, rng, 20 + n, heads, dim, t=t)
    v[20 + 70, 0, 3], v[20 + 71, 1, dim - 1], k[20 + 90, 0, 5], v[20 + n - 1, 0, 0] = float("inf"), float("nan"), float("nan"), float("-inf")
    v[20 + 149, 1] = float("nan")
    k[20 + 140, 1] = float("inf")
    y = torch.zeros_like(q, device="cuda:0")
    for workspace in (aqd.ATTN_WORKSPACE_BYTES, 0):
        run_attn(torch, q.cuda(), k.cuda(), v.cuda(), qs, ks, True, t, y, workspace)
        got = y.double().cpu().numpy()
        clean = [x.double().numpy().copy() for x in (k, v)]
        for x in clean:
            x[~np.isfinite(x)] = 0
        seq = got[20:]
        ok = np.ones((n, heads, per, dim), bool)
        i = np.arange(n)
        ok[i >= 70, 0, :, 3] = False
        ok[i >= 71, 1, :, dim - 1] = False
        ok[i >= 90, 0] = False
        ok[i >= 140, 1] = False
        ok = ok.reshape(n, heads * per, dim)
        assert np.isfinite(seq[ok]).all() and np.isfinite(got[:20]).all()
        one = seq.reshape(n, heads, per, dim)
        assert (one[70:90, 0, :, 3] == np.inf).all() and np.isnan(one[71:, 1, :, dim - 1]).all() and np.isnan(one[90:, 0]).all()
        want = plain.attention(q[20:].double().numpy(), clean[0][20:], clean[1][20:], dim ** -0.5, True)[0]
        filled = np.where(ok, seq, want)
        # queries past the first hidden key's own see it: they were compared above
        for h, end in ((0, 90), (1, 140)):
            rows = slice(h * per, (h + 1) * per)
            check_attention(filled[:end, rows], q[20:20 + end, rows].double().numpy(), clean[0][20:20 + end, h:h + 1], clean[1][20:20 + end, h:h + 1],
                            dim ** -0.5, True, t)


def test_attn_starts_that_leave_the_rows():
    """Starts are bounded by the rows there are; a sequence that ends before it starts is empty."""
    import torch
    rng = np.random.Generator(np.random.PCG64(77))
    t, dim = "bf16", 64
    q, k, v = [reals(torch, rng, 30, 2, dim, t=t) for _ in range(3)]
    y = torch.full_like(q, 77, device="cuda:0")
    run_attn(torch, q.cuda(), k.cuda(), v.cuda(), [-5, 12, 10, 20, 99], [-3, 10, 12, 5, 2 ** 31 - 1], False, t, y, max_queries=10)
    got = y.double().cpu().numpy()
    n64 = [x.double().numpy() for x in (q, k, v)]
    for a, b, c, d in ((0, 10, 0, 10), (20, 30, 5, 30)):
        check_attention(got[a:b], n64[0][a:b], n64[1][c:d], n64[2][c:d], dim ** -0.5, False, t)
    # the first sequence's rows 10 and 11 are past max_queries; the third's keys end before they start
    assert not got[10:20].any()

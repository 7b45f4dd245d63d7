"""The attention operators at the ends of what their arguments may be: keys next to 2^31, values and scores next to fp32's largest
numbers. Tolerances: test_gpu_attention.py."""
import numpy as np
import pytest

import attention_plain as plain
from paper_2007_06919_amd import aqd
from test_gpu_attention import OFFSET, U, Sequences, check_attention, close, reals, run_attn, run_qattn, strides

pytestmark = pytest.mark.gpu

MOST_KEYS = 2 ** 31 - 1 - 65536


def test_qattn_of_as_many_tokens_as_there_may_be():
    """One page again and again, and another at the end, whose tokens have nearly all of the weight: e^40 each, the others 1."""
    import torch
    dim, page, last, t = 64, 256, 100, "bf16"
    c = aqd.QcacheDesc(1, dim, 64, page, 2)
    rng = np.random.Generator(np.random.PCG64(31))
    k, v = np.zeros((2 * page, 1, dim), np.float32), rng.standard_normal((2 * page, 1, dim)).astype(np.float32)
    k[page:] = 0.625                                                  # a group's largest element is kept: -5/64 in bf16, and -8
    v[page:] += 3
    cache = np.zeros((2, 1, plain.block_bytes(dim, 64, page)), np.uint8)
    slots = np.arange(2 * page)
    plain.write(cache, slots, k, v, 1, dim, 64, page)
    kr, vr, ks, vs = plain.read(cache, slots, 1, dim, 64, page)
    tables = torch.zeros(1, -(-MOST_KEYS // page), dtype=torch.int32, device="cuda:0")
    tables[0, -last:] = 1
    q = torch.ones(1, 1, dim).bfloat16()
    y = torch.zeros_like(q, device="cuda:0")
    run_qattn(torch, c, torch.from_numpy(cache).cuda(), tables, [MOST_KEYS], q.cuda(), None, 1, t, y, scale=1.0)
    end = MOST_KEYS - (MOST_KEYS - 1) // page * page                  # tokens of the last page
    mean = ((last - 1) * vr[page:].sum(0) + vr[page:page + end].sum(0)) / ((last - 1) * page + end)
    size = vs[page:].max(0)                                           # a value is 8 of it at most, and 280 in the sum of code + 128
    # the others: 2^31 of e^-40 by the last pages' 25000
    others = 2.0 ** 31 * np.exp(-40.0) / (last * page) * 2 * np.abs(vr).max()
    close(y.double().cpu().numpy()[0], mean, (plain.HALF[t] + 8 * U) * 8 * size + (last * page / 8 + 8) * 2 * U * OFFSET[t] * size +
          1.01 * plain.HALF[t] * np.abs(mean) + others)


@pytest.mark.parametrize("causal", [True, False])
def test_attn_of_as_many_keys_as_there_may_be(causal):
    import torch
    dim, t = 8, "bf16"
    rng = np.random.Generator(np.random.PCG64(32))
    k = torch.zeros(MOST_KEYS, 1, dim, dtype=torch.bfloat16, device="cuda:0")   # and the values
    tail = 1 + reals(torch, rng, 5, 1, dim, t=t, scale=0.125)
    k[-5:] = tail.cuda()
    q = 5 + reals(torch, rng, 2, 3, dim, t=t, scale=0.125)
    y = torch.zeros_like(q, device="cuda:0")
    run_attn(torch, q.cuda(), k, k, [0, 2], [0, MOST_KEYS], causal, t, y, scale=1.0)
    del k
    got = y.double().cpu().numpy()
    for i in range(2):
        seen = tail[:4 + i if causal else 5].double().numpy()
        want, rest, size, most = plain.attention(q[i:i + 1].double().numpy(), seen, seen, 1.0, False)
        others = 2.0 ** 31 * np.exp(-(q[i].double().numpy() @ seen[:, 0].T).max())   # their share of the weight, and no value
        close(got[i], want[0], (dim / 8 + 2) * 2 * U * most[0][:, None] * rest[0] + (plain.HALF[t] + 24 * U + others) * size[0] + 1.01 * plain.HALF[t] * np.abs(want[0]))


@pytest.mark.parametrize("dim, heads, per, nq, nk", [(128, 1, 2, [3, 70], [900, 70]), (64, 2, 1, [1], [3000]), (256, 1, 1, [40], [40]), (72, 1, 3, [5], [2500])])
@pytest.mark.parametrize("size", [1e34, 7e37])
def test_attn_of_values_next_to_the_largest(size, dim, heads, per, nq, nk):
    import torch
    t = "bf16"
    rng = np.random.Generator(np.random.PCG64(34 + dim))
    qs, ks = [0] + list(np.cumsum(nq)), [0] + list(np.cumsum(nk))
    q, k = reals(torch, rng, qs[-1], heads * per, dim, t=t), reals(torch, rng, ks[-1], heads, dim, t=t)
    v = torch.from_numpy(rng.uniform(-4.5, 4.5, (ks[-1], heads, dim)) * size)
    v[..., 0] = 4.5 * size
    v[..., 32:] = torch.from_numpy(rng.standard_normal(v[..., 32:].shape))
    v = v.bfloat16()
    for workspace in (aqd.ATTN_WORKSPACE_BYTES, 0):
        for causal in (True, False):
            y = torch.zeros_like(q, device="cuda:0")
            run_attn(torch, q.cuda(), k.cuda(), v.cuda(), qs, ks, causal, t, y, workspace)
            got = y.double().cpu().numpy()
            for b in range(len(nq)):
                a, z = slice(qs[b], qs[b + 1]), slice(ks[b], ks[b + 1])
                check_attention(got[a], q[a].double().numpy(), k[z].double().numpy(), v[z].double().numpy(), dim ** -0.5, causal, t, name=f"sequence {b}")


@pytest.mark.parametrize("heads, dim, group, per, lengths, counts", [
    (2, 128, 32, 4, [500, 3], [1, 1]), (1, 64, 64, 3, [9000], [1]), (1, 64, 32, 8, [700, 40], [9, 5]), (1, 256, 32, 2, [300], [20]), (2, 256, 128, 1, [90], [1]),
    (1, 128, 64, 16, [40] * 9 + [5000], [1] * 10),
])
@pytest.mark.parametrize("size", [1e29, 1e33, 7e37])
def test_qattn_of_values_next_to_the_largest(size, heads, dim, group, per, lengths, counts):
    """A result is never larger than its values, whatever the sums before the division by the weights. The last group has values
    of ordinary size."""
    import torch
    page, t = 16, "bf16"
    s = Sequences(torch, 33, lengths, heads, dim, group, page)
    for b, v in enumerate(s.v):
        big = s.rng.uniform(-4.5, 4.5, v.shape) * size
        if dim > group:
            big[..., -group:] = s.rng.standard_normal(big[..., -group:].shape)
        big[len(big) // 2:, ..., 0] = 4.5 * size                      # all of one sign
        plain.write(s.cache, s.slots(b), s.k[b].astype(np.float32), big.astype(np.float32), *s.shape)
        s.k[b], s.v[b], s.ks[b], s.vs[b] = plain.read(s.cache, s.slots(b), *s.shape)
    start = [0] + list(np.cumsum(counts))
    q = reals(torch, s.rng, start[-1], heads * per, dim, t=t)
    cache, tables = torch.from_numpy(s.cache).cuda(), torch.from_numpy(s.tables).cuda()
    for workspace in (aqd.ATTN_WORKSPACE_BYTES, 0):
        y = torch.zeros_like(q, device="cuda:0")
        run_qattn(torch, s.c, cache, tables, lengths, q.cuda(), start, max(counts), t, y, workspace)
        s.check(y.double().cpu().numpy(), q, start, t)


@pytest.mark.parametrize("count", [1, 20])
def test_qattn_of_large_values_with_hardly_any_weight_fp16(count):
    """Two tokens: 2.9e38 with the weight e^-80, and next to nothing with the rest. What is left of the first is a number in fp16. (Products of a weight
    and a scale: within half a step, or 2^-24 of the row's largest, times a code.)"""
    import torch
    dim, page, t = 64, 16, "f16"
    c = aqd.QcacheDesc(1, dim, 32, page, 2)
    n = count + 1
    k, v = np.zeros((n, 1, dim), np.float32), np.full((n, 1, dim), 1e-20, np.float32)
    k[1:, :, :32] = 2.5
    v[0] = 2.9e38 * np.linspace(0.5, 1, dim)
    cache = np.zeros((2, 1, plain.block_bytes(dim, 32, page)), np.uint8)
    plain.write(cache, np.arange(n), k, v, 1, dim, 32, page)
    kr, vr, ks, vs = plain.read(cache, np.arange(n), 1, dim, 32, page)
    q = torch.ones(count, 1, dim).half()
    y = torch.zeros_like(q, device="cuda:0")
    run_qattn(torch, c, torch.from_numpy(cache).cuda(), torch.arange(2, dtype=torch.int32, device="cuda:0").view(1, 2), [n], q.cuda(), [0, count], count, t, y,
              scale=1.0)
    got = y.double().cpu().numpy()
    for i in range(count):
        m, one = i + 2, q[i:i + 1].double().numpy()
        want, rest, size, most = plain.attention(one, kr[:m], vr[:m], 1.0, False, OFFSET[t] * ks[:m], OFFSET[t] * vs[:m])
        weights = plain.attention(one, kr[:m], vr[:m], 1.0, False)[2]
        close(got[i:i + 1], want, (dim / 8 + 2) * 2 * U * most[..., None] * rest + (plain.HALF[t] + 8 * U) * weights + (m / 8 + 8) * 2 * U * size +
              1.01 * plain.HALF[t] * np.abs(want) + plain.LEAST[t] + m * 2.0 ** -24 * weights.max() * 8)


@pytest.mark.parametrize("scale", [0.0, 1e-32, -1e-32, 1e-39])
def test_small_scales_of_large_scores(scale):
    """Products of queries and keys of about 2^106: a scale of 0 makes every weight the same, smaller ones than 2^-100 count as they are."""
    import torch
    dim, page, t = 64, 16, "bf16"
    rng = np.random.Generator(np.random.PCG64(35))
    big = 2.0 ** 52
    q, k = [reals(torch, rng, n, h, dim, t=t, scale=big) for n, h in ((20, 4), (90, 2))]
    v = reals(torch, rng, 90, 2, dim, t=t)
    n64 = [x.double().numpy() for x in (q, k, v)]
    c = aqd.QcacheDesc(2, dim, 32, page, 6)
    cache = torch.zeros(aqd.qcache_bytes(c), dtype=torch.uint8, device="cuda:0")
    slots = torch.arange(90, dtype=torch.int32, device="cuda:0")
    kd, vd = k.cuda(), v.cuda()
    aqd.qcache_write(c, 90, aqd.BF16, kd, *strides(kd), vd, *strides(vd), slots, cache)
    kr, vr, ks, vs = plain.read(cache.cpu().numpy().reshape(6, 2, -1), np.arange(90), 2, dim, 32, page)
    y = torch.zeros_like(q, device="cuda:0")
    for causal in (True, False):
        run_attn(torch, q.cuda(), kd, vd, [0, 20], [0, 90], causal, t, y, scale=scale)
        check_attention(y.double().cpu().numpy(), *n64, scale, causal, t, name=f"prompt {causal}")
    for count in (20, 1):
        some = q[:count].cuda()
        run_qattn(torch, c, cache, slots[:6].view(1, 6), [90], some, [0, count], count, t, y[:count], scale=scale)
        check_attention(y[:count].double().cpu().numpy(), n64[0][:count], kr, vr, scale, True, t, OFFSET[t] * ks, OFFSET[t] * vs, name=f"cache {count}")

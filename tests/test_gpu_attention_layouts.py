"""Queries, keys, values and results that alternate head by head in one row, [tokens][heads][4][dim] with something between the rows: every
call has the bits that it has on packed tensors, and leaves the rest of the rows as it was."""
import numpy as np
import pytest

from attention_plain import DTYPE
from paper_2007_06919_amd import aqd
from test_gpu_attention import TYPES, make_table, run_attn, run_heads, run_qattn, strides

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("t", ["f16", "bf16"])
@pytest.mark.parametrize("pad", [0, 24])
@pytest.mark.parametrize("tokens", [1, 2, 37])
@pytest.mark.parametrize("heads, dim", [(1, 128), (2, 64), (8, 128)])
def test_heads_that_alternate(heads, dim, tokens, pad, t):
    import torch
    rng = np.random.Generator(np.random.PCG64(dim + tokens))
    rows = torch.from_numpy(rng.standard_normal((tokens, heads * 4 * dim + pad))).to(DTYPE[t]).cuda()
    four = rows[:, :heads * 4 * dim].unflatten(1, (heads, 4, dim))
    q, k, v, y = (four[:, :, i] for i in range(4))
    packed = [x.contiguous() for x in (q, k, v)]
    before = rows.clone()

    def unchanged(but):
        now, old = rows.clone(), before.clone()
        for x in (now, old):
            x[:, :heads * 4 * dim].unflatten(1, (heads, 4, dim))[:, :, but] = 0
        assert torch.equal(now, old)
        before.copy_(rows)

    table, position = torch.from_numpy(make_table(50, dim)).cuda(), torch.arange(tokens, dtype=torch.int32, device="cuda:0")
    for a, b in ((q, k), packed[:2]):
        run_heads(torch, a, b, None, None, table, position, dim, aqd.PAIRS_HALVES, t, a, b)
    assert torch.equal(q, packed[0]) and torch.equal(k, packed[1])
    unchanged([0, 1])

    want = torch.zeros_like(packed[0])
    run_attn(torch, *packed, [0, tokens], [0, tokens], True, t, want)
    run_attn(torch, q, k, v, [0, tokens], [0, tokens], True, t, y)
    assert torch.equal(y, want)
    unchanged([3])

    c = aqd.QcacheDesc(heads, dim, 32, 16, 4)
    caches = [torch.zeros(aqd.qcache_bytes(c), dtype=torch.uint8, device="cuda:0") for _ in range(2)]
    for cache, a, b in ((caches[0], k, v), (caches[1], *packed[1:])):
        aqd.qcache_write(c, tokens, TYPES[t], a, *strides(a), b, *strides(b), position, cache)
    assert torch.equal(*caches)
    tables = torch.arange(4, dtype=torch.int32, device="cuda:0").view(1, 4)
    run_qattn(torch, c, caches[0], tables, [tokens], packed[0], [0, tokens], tokens, t, want)
    run_qattn(torch, c, caches[0], tables, [tokens], q, [0, tokens], tokens, t, y)
    assert torch.equal(y, want)
    unchanged([3])
    for a, b in ((k, v), packed[1:]):
        aqd.qcache_read(c, tokens, TYPES[t], caches[0], position, a, *strides(a), b, *strides(b))
    assert torch.equal(k, packed[1]) and torch.equal(v, packed[2])
    unchanged([1, 2])


@pytest.mark.parametrize("t, dim", [("bf16", 128), ("f16", 64), ("bf16", 200)])
def test_first_tokens_of_a_large_buffer(t, dim):
    """Keys and values [heads][tokens][dim] with room for so many that the heads are more than 2^26 elements apart, and none, one and two tokens in
    it."""
    import torch
    rng = np.random.Generator(np.random.PCG64(dim))
    heads, room = 3, -(-((1 << 26) + 4096) // dim)
    k, v = [torch.full((heads, room, dim), float("nan"), dtype=DTYPE[t], device="cuda:0") for _ in range(2)]
    for n in (0, 1, 2):
        q, a, b = [torch.from_numpy(rng.standard_normal((m, h, dim))).to(DTYPE[t]).cuda() for m, h in ((2, 6), (n, heads), (n, heads))]
        k[:, :n], v[:, :n] = a.transpose(0, 1), b.transpose(0, 1)
        want, y = torch.full_like(q, 7), torch.full_like(q, 7)
        for causal in (True, False):
            run_attn(torch, q, a, b, [0, 2], [0, n], causal, t, want)
            run_attn(torch, q, k[:, :n].transpose(0, 1), v[:, :n].transpose(0, 1), [0, 2], [0, n], causal, t, y)
            assert torch.equal(y, want), (n, causal)

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

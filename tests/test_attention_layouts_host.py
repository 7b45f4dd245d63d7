"""Layouts of heads and tokens that the attention calls take or refuse: the checks come from the host before any launch. What they take is
launched, so where there is a GPU, calls with addresses of nothing are left out (test_gpu_attention_layouts.py has them with memory)."""
import ctypes
import random

import pytest
import torch

from paper_2007_06919_amd import aqd

NO_GPU = pytest.mark.skipif(torch.cuda.device_count() > 0, reason="addresses of nothing would be launched")
AT = 1 << 40


def status(call, *args, **kw):
    try:
        call(*args, **kw)
    except aqd.AqdError as e:
        return e.status
    return aqd.AQD_OK


def taken(s):
    """Without a GPU a launch fails."""
    return s in (aqd.AQD_OK, aqd.AQD_ERR_DEVICE)


def heads_in_place(tokens, heads, k_heads, dim, q, q_token, q_head, k, k_token, k_head):
    return status(aqd.heads_run, tokens, heads, k_heads, dim, 0, aqd.PAIRS_HALVES, aqd.BF16, 0, 1e-6, q, q_token, q_head, k, k_token, k_head, None, None, None, None,
                  q, q_token, q_head, k, k_token, k_head, 0)


def read_into(tokens, heads, dim, k, k_token, k_head, v, v_token, v_head):
    c = aqd.QcacheDesc(heads, dim, 32, 16, 4)
    return status(aqd.qcache_read, c, tokens, aqd.BF16, 1 << 20, 1 << 24, k, k_token, k_head, v, v_token, v_head, 0)


@NO_GPU
@pytest.mark.parametrize("tokens", [1, 2, 4, 1000])
@pytest.mark.parametrize("pad", [0, 64, 24])
@pytest.mark.parametrize("heads", [1, 2, 8])
def test_heads_whose_queries_keys_and_values_alternate(heads, pad, tokens):
    """[tokens][heads][3][dim] and `pad` elements between the rows."""
    dim, head = 64, 3 * 64
    token = heads * head + pad
    q, k, v = (AT + 2 * dim * i for i in range(3))
    assert taken(heads_in_place(tokens, heads, heads, dim, q, token, head, k, token, head))
    assert taken(read_into(tokens, heads, dim, k, token, head, v, token, head))
    # half a head into the other's, from either side; the next row's first
    for at in (q + dim, q - dim, q + 2 * (token - dim // 2) * (tokens > 1)):
        assert heads_in_place(tokens, heads, heads, dim, q, token, head, at, token, head) == aqd.AQD_ERR_INVALID
        assert read_into(tokens, heads, dim, q, token, head, at, token, head) == aqd.AQD_ERR_INVALID


@NO_GPU
@pytest.mark.parametrize("tokens", [1, 2, 5])
def test_one_key_head_in_a_gap_of_the_queries(tokens):
    """Rows of q0, k, q1, other things: one key head has no head stride."""
    dim, head = 64, 128
    assert taken(heads_in_place(tokens, 2, 1, dim, AT, 300, head, AT + 2 * dim, 300, 7))
    assert heads_in_place(tokens, 2, 1, dim, AT, 300, head, AT + 2 * dim + 2, 300, 7) == aqd.AQD_ERR_INVALID


@NO_GPU
def test_tensors_that_meet_are_refused_and_others_are_not():
    """Against the elements themselves: what meets is refused, what does not and has one make of rows is taken."""
    rng = random.Random(1)
    dim, met, free = 2, 0, 0
    for _ in range(4000):
        tokens, heads = rng.randint(1, 4), rng.randint(1, 4)
        k_heads = heads if rng.random() < 0.7 else rng.randint(1, 4)
        head = rng.randint(dim, 9)
        token = (max(heads, k_heads) - 1) * head + dim + rng.randint(0, 9)
        if rng.random() < 0.3:       # [heads][tokens]
            token, head = head, (tokens - 1) * head + dim + rng.randint(0, 9)
        same = rng.random() < 0.8
        k_token, k_head = (token, head) if same else (token + rng.randint(0, 3), head)
        gap = rng.randint(-40, 40)
        a = {t * token + h * head + c for t in range(tokens) for h in range(heads) for c in range(dim)}
        b = {gap + t * k_token + h * k_head + c for t in range(tokens) for h in range(k_heads) for c in range(dim)}
        if len(a) < tokens * heads * dim or len(b) < tokens * k_heads * dim:
            continue
        got = heads_in_place(tokens, heads, k_heads, dim, AT, token, head, AT + 2 * gap, k_token, k_head)
        what = (tokens, heads, k_heads, token, head, k_token, k_head, gap)
        if a & b:
            assert got == aqd.AQD_ERR_INVALID, what
            met += 1
        elif same and heads == k_heads:
            assert taken(got), what
            free += 1
    assert met > 500 and free > 500


@NO_GPU
@pytest.mark.parametrize("token, head", [(0, 0), (1, 1), (-5, 1 << 62)])
def test_tensors_without_tokens_have_no_strides(token, head):
    """As torch's of an empty numpy array, whose strides are 0."""
    c, none = aqd.QcacheDesc(2, 64, 32, 16, 4), (None, token, head)
    for batch in (0, 1):
        assert status(aqd.attn_run, batch, 4, 2, 64, 0, 10, 0, 10, True, aqd.BF16, 0.1, *none, AT, 128, 64, AT, 128, 64, AT, AT, *none, stream=0) == aqd.AQD_OK
        assert status(aqd.qattn_run, c, batch, 4, 0, 0, 10, aqd.BF16, 0.1, *none, AT, AT, AT, 1, AT, *none, stream=0) == aqd.AQD_OK
    # queries without a key have zeros
    q, y, start = AT, 2 * AT, 3 * AT
    assert taken(status(aqd.attn_run, 1, 4, 2, 64, 2, 0, 2, 0, True, aqd.BF16, 0.1, q, 256, 64, *none, *none, start, start, y, 256, 64, stream=0))


@pytest.mark.parametrize("keys", [0, 1, 2, 3])
def test_few_keys_of_a_large_buffer(keys):
    """[heads][131072 tokens][128] with hardly any token in it: the heads are far apart, the tokens are not."""
    token, head = 128, 131072 * 128
    d = aqd.AttnDesc(1, 8, 8, 128, 1, keys, 1, keys, 1, aqd.BF16, 0.1, 8 * 128, 128, token, head, token, head, 8 * 128, 128)
    size = ctypes.c_size_t(7)
    assert aqd.lib().aqd_attn_workspace(ctypes.byref(d), ctypes.byref(size)) == aqd.AQD_OK and size.value == 0


@pytest.mark.parametrize("keys", [0, 1])
def test_a_single_key_has_no_token_stride(keys):
    for token in (0, -1, 1, (1 << 26) + 1, 1 << 60):
        d = aqd.AttnDesc(1, 8, 8, 128, 1, keys, 1, keys, 1, aqd.BF16, 0.1, 8 * 128, 128, token, 1 << 27, token, 128, 8 * 128, 128)
        size = ctypes.c_size_t(7)
        assert aqd.lib().aqd_attn_workspace(ctypes.byref(d), ctypes.byref(size)) == aqd.AQD_OK and size.value == 0

"""The attention operators in plain form on the host: numpy in 64 bits where numbers are computed, the
definition's fp32 steps where codes are chosen, the cache's layout channel by channel. No GPU, none of the library."""
import numpy as np
import torch

HALF = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}   # half a step, relative
LEAST = {"f32": 2.0 ** -150, "f16": 2.0 ** -25, "bf16": 2.0 ** -134}   # half the smallest number
DTYPE = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def heads(x, weight, eps, table, position, rot, halves):
    """(result, |n_a| + |n_b| of each channel's pair) for x [tokens][heads][dim] in float64."""
    n = x.copy()
    if weight is not None:
        n = n / np.sqrt((n * n).mean(-1, keepdims=True) + eps) * weight
    y, size = n.copy(), np.abs(n)
    for i in range(rot // 2):
        a, b = (i, i + rot // 2) if halves else (2 * i, 2 * i + 1)
        c, s = table[position, i][:, None], table[position, rot // 2 + i][:, None]
        y[..., a] = n[..., a] * c - n[..., b] * s
        y[..., b] = n[..., b] * c + n[..., a] * s
        size[..., a] = size[..., b] = np.abs(n[..., a]) + np.abs(n[..., b])
    return y, size


def quantise(x, group):
    """(codes uint8 [..., dim], scales float32 that bf16 holds [..., dim / group]) of float32 x."""
    u = x.reshape(x.shape[:-1] + (x.shape[-1] // group, group))
    top, low = u.max(-1), u.min(-1)
    a = np.where(top >= -low, top, low).astype(np.float32)
    s = torch.from_numpy(a * np.float32(-0.125)).bfloat16().float().numpy()
    s[np.abs(s) < 2.0 ** -119] = 0
    bad = ~np.isfinite(u).all(-1)
    with np.errstate(all="ignore"):
        r = np.where((s == 0) | bad, np.float32(0), np.float32(1) / s).astype(np.float32)
        c = np.clip(np.rint(u * r[..., None]), -8, 7)
    c[bad] = 0
    s[bad] = np.nan
    return (c.reshape(x.shape) + 8).astype(np.uint8), s


def places(heads, dim, group, page):
    """Of each token and channel of a block: byte and shift of the key's and the value's code, and the indices of the keys'
    and values' scales among the block's 16-bit numbers."""
    t, c = np.arange(page)[:, None], np.arange(dim)[None, :]
    w, nibble = c // 8, c % 8 // 2 + c % 2 * 4
    key = t * (dim // 2) + 4 * (w % 4 * (dim // 32) + w // 4) + nibble // 2
    unit = ((t // 4 * 16 + c % 16) * (dim // 64) + c // 64) * 4 + t % 4
    n = c % 64 // 16
    value = page * dim // 2 + 2 * unit + n // 2
    g = np.arange(dim // group)[None, :]
    scale = page * dim // 2 + t * (dim // group) + g
    return key, nibble % 2 * 4 + 0 * t, value, n % 2 * 4 + 0 * t, scale, scale + page * (dim // group)


def block_bytes(dim, group, page):
    return page * (dim + 4 * (dim // group))


def write(cache, slots, k, v, heads, dim, group, page):
    """Rows k, v float32 [tokens][heads][dim] into cache uint8 [pages][heads][bytes], in place."""
    key, ks, value, vs, kscale, vscale = places(heads, dim, group, page)
    for codes_at, shift, scale_at, x in ((key, ks, kscale, k), (value, vs, vscale, v)):
        codes, scales = quantise(x, group)
        bits = torch.from_numpy(scales).bfloat16().view(torch.int16).numpy().view(np.uint16)
        bits = np.where(np.isnan(scales), np.uint16(0x7FC0), bits)
        for t, slot in enumerate(slots):
            if not 0 <= slot < len(cache) * page:
                continue
            for h in range(heads):
                block, i = cache[slot // page, h], slot % page
                np.bitwise_and.at(block, codes_at[i], (0xF0 >> shift[i]).astype(np.uint8))
                np.bitwise_or.at(block, codes_at[i], codes[t, h] << shift[i].astype(np.uint8))
                block.view(np.uint16)[scale_at[i]] = bits[t, h]


def read(cache, slots, heads, dim, group, page):
    """(keys, values, their scales of each channel) float64 [tokens][heads][dim] of the slots, which lie in the cache."""
    key, ks, value, vs, kscale, vscale = places(heads, dim, group, page)
    out = []
    blocks = cache[slots // page]                                # [tokens][heads][bytes]
    i = slots % page
    numbers = torch.from_numpy(np.ascontiguousarray(blocks).view(np.int16)).view(torch.bfloat16).double().numpy()
    sizes = []
    for at, shift, scale_at in ((key, ks, kscale), (value, vs, vscale)):
        code = np.take_along_axis(blocks, at[i][:, None, :].repeat(heads, 1), 2) >> shift[i][:, None, :] & 15
        scale = np.take_along_axis(numbers, scale_at[i][:, None, :].repeat(heads, 1), 2).repeat(group, -1)
        out.append((code.astype(np.float64) - 8) * scale)
        sizes.append(np.abs(scale))
    return out[0], out[1], sizes[0], sizes[1]


def attention(q, k, v, scale, causal, k_size=None, v_size=None):
    """One sequence: q [n][q_heads][dim], k and v [m][heads][dim] in float64. Returns the result, its sensitivity to the scores (what an
    error e of every score changes at most: e * this), and the weighted sum of v_size (of |v| without it)."""
    n, m, per = q.shape[0], k.shape[0], q.shape[1] // k.shape[1]
    y, rest, size = np.zeros_like(q), np.zeros(q.shape), np.zeros_like(q)
    most = np.zeros(q.shape[:2])
    v_size = np.abs(v) if v_size is None else v_size
    k_size = np.abs(k) if k_size is None else k_size
    for i in range(n):
        seen = max(0, m - n + 1 + i) if causal else m
        if not seen:
            continue
        for h in range(q.shape[1]):
            kv = h // per
            s = k[:seen, kv] @ q[i, h] * scale
            p = np.exp(s - s.max())
            p /= p.sum()
            y[i, h] = p @ v[:seen, kv]
            size[i, h] = p @ v_size[:seen, kv]
            rest[i, h] = p @ np.abs(v[:seen, kv] - y[i, h])
            most[i, h] = (k_size[:seen, kv] @ np.abs(q[i, h])).max() * abs(scale)
    return y, rest, size, most

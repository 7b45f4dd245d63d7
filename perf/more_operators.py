"""Performance cases of the attention operators: norms of query and key heads with the
rotation by position in the same pass (``heads``), a cache of keys and values that is
quantised to 4 bits as it is written and read back (``cache``), attention over such a
cache (``qattn``), and attention over whole prompts of packed sequences (``attn``).

``run`` computes an operator in elementary torch operations in 32 bits, or, where
``own`` is true, by the library's entry points. Both read the same packed cache.

The cache: pages of ``page`` tokens, a page has one block per head: the tokens' key
codes, then their value codes, then the keys' scales, then the values' (bf16, one per
group of channels). A code c stands for scale * (c - 8).
"""
from __future__ import annotations

import random

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
LEAST = 2.0 ** -119                # scales below are 0
EPS = 1e-6
WORKSPACE = 64 << 20               # what a program keeps for partial results, one per stream

MOST_HEADS = 16384 * 40 * 128      # elements of the largest listed case of each operator
MOST_CACHE = 16384 * 8 * 128
MOST_QATTN = 3 * 120000 * 8 * 128
MOST_ATTN = 16384 * 16384 // 2 * 32 * 128


def listed():
    return [
        # one token of one sequence that decodes, slices of a joint projection's row: what a call costs at least
        {"name": "heads_1x32+8x128_bf16", "op": "heads", "tokens": 1, "q_heads": 32, "k_heads": 8, "dim": 128, "rot": 128,
         "pairs": "halves", "type": "bf16", "pad": 1024, "norm": True},
        # odd sizes, fp32, neighbouring channels turned, the last quarter of a head not
        {"name": "heads_1003x7+1x80_f32", "op": "heads", "tokens": 1003, "q_heads": 7, "k_heads": 1, "dim": 80, "rot": 60,
         "pairs": "neighbours", "type": "f32", "pad": 0, "norm": True},
        # a batch of prompts
        {"name": "heads_16384x32+8x128_bf16", "op": "heads", "tokens": 16384, "q_heads": 32, "k_heads": 8, "dim": 128, "rot": 128,
         "pairs": "halves", "type": "bf16", "pad": 1024, "norm": True},
        # 64 sequences that decode together write a token each
        {"name": "cache_64x8x128_g32_bf16", "op": "cache", "tokens": 64, "heads": 8, "dim": 128, "group": 32, "page": 16, "run": 1,
         "type": "bf16", "pad": 4096},
        # a batch of prompts is written, and read back for the next chunk of the prompts
        {"name": "cache_16384x8x128_g64_bf16", "op": "cache", "tokens": 16384, "heads": 8, "dim": 128, "group": 64, "page": 64,
         "run": 2048, "type": "bf16", "pad": 4096},
        # one sequence decodes
        {"name": "qattn_1x1500_32:8x128_g32_bf16", "op": "qattn", "batch": 1, "low": 1500, "high": 1500, "salt": 1, "q_heads": 32,
         "heads": 8, "dim": 128, "group": 32, "page": 16, "tokens": 1, "type": "bf16"},
        # 64 sequences of unequal lengths decode together
        {"name": "qattn_64x8192_32:8x128_g32_bf16", "op": "qattn", "batch": 64, "low": 700, "high": 8192, "salt": 2, "q_heads": 32,
         "heads": 8, "dim": 128, "group": 32, "page": 16, "tokens": 1, "type": "bf16"},
        # sixteen sequences with four draft tokens each, half precision, small heads
        {"name": "qattn_16x4x2500_24:3x64_g64_f16", "op": "qattn", "batch": 16, "low": 5, "high": 2500, "salt": 3, "q_heads": 24,
         "heads": 3, "dim": 64, "group": 64, "page": 32, "tokens": 4, "type": "f16"},
        # three very long sequences
        {"name": "qattn_3x120000_64:8x128_g128_bf16", "op": "qattn", "batch": 3, "low": 100000, "high": 120000, "salt": 4, "q_heads": 64,
         "heads": 8, "dim": 128, "group": 128, "page": 256, "tokens": 1, "type": "bf16"},
        # a short chunk of a prompt behind what was read before
        {"name": "attn_100of1337_12:4x64_f16", "op": "attn", "batch": 1, "low": 1337, "high": 1337, "salt": 5, "part": 100, "q_heads": 12,
         "heads": 4, "dim": 64, "causal": True, "type": "f16", "pad": 0},
        # prompts of unequal lengths packed into one batch, slices of a joint projection's rows
        {"name": "attn_17x2048_32:8x128_bf16", "op": "attn", "batch": 17, "low": 40, "high": 2048, "salt": 6, "part": 0, "q_heads": 32,
         "heads": 8, "dim": 128, "causal": True, "type": "bf16", "pad": 2048},
        # one long prompt
        {"name": "attn_1x16384_32:8x128_bf16", "op": "attn", "batch": 1, "low": 16384, "high": 16384, "salt": 7, "part": 0, "q_heads": 32,
         "heads": 8, "dim": 128, "causal": True, "type": "bf16", "pad": 0},
    ]


def _spread(rng, low, high):
    """A size between low and high, even over its logarithm."""
    return max(low, min(high, int(round(low * (high / low) ** rng.random()))))


def draw(rng):
    op = rng.choice(["heads", "cache", "qattn", "qattn", "attn", "attn"])
    kind = rng.choice(["bf16", "bf16", "f16"])
    per = rng.choice([1, 2, 3, 4, 7, 8, 16])
    heads = rng.choice([1, 2, 3, 4, 8, 8, 16])
    if op == "heads":
        kind = rng.choice(["bf16", "bf16", "f16", "f32"])
        dim = rng.choice([64, 128, 128, 256, 2 * rng.randrange(16, 128)])
        while True:
            tokens = _spread(rng, 1, 32768)
            if tokens * heads * (per + 1) * dim <= MOST_HEADS:
                break
            heads, per = max(1, heads // 2), max(1, per // 2)
        return {"op": op, "tokens": tokens, "q_heads": heads * per, "k_heads": heads, "dim": dim,
                "rot": dim if rng.random() < 0.7 else 2 * rng.randrange(1, dim // 2), "pairs": rng.choice(["halves", "halves", "neighbours"]),
                "type": kind, "pad": rng.choice([0, heads * dim, rng.randrange(1, 64)]), "norm": rng.random() < 0.8}
    dim = rng.choice([64, 128, 128, 256])
    group = rng.choice([g for g in (32, 64, 128) if g <= dim])
    page = rng.choice([16, 16, 32, 64, 128, 256])
    if op == "cache":
        kind = rng.choice(["bf16", "bf16", "f16", "f32"])
        while True:
            tokens = _spread(rng, 1, 65536)
            if tokens * heads * dim <= MOST_CACHE:
                break
            heads = max(1, heads // 2)
        return {"op": op, "tokens": tokens, "heads": heads, "dim": dim, "group": group, "page": page,
                "run": rng.choice([1, 1000, _spread(rng, 1, tokens)]), "type": kind, "pad": rng.choice([0, heads * dim * per, rng.randrange(1, 64)])}
    salt = rng.randrange(1 << 30)
    if op == "qattn":
        while True:
            batch, high = _spread(rng, 1, 256), _spread(rng, 1, 131072)
            if batch * high * heads * dim <= MOST_QATTN:
                break
        return {"op": op, "batch": batch, "low": rng.choice([0, high // 2, high]), "high": high, "salt": salt, "q_heads": heads * per,
                "heads": heads, "dim": dim, "group": group, "page": page, "tokens": rng.choice([1, 1, 1, 2, 4, 7]), "type": kind}
    while True:
        batch, high = _spread(rng, 1, 64), _spread(rng, 1, 16384)
        if batch * high * high // 2 * heads * per * dim <= MOST_ATTN and batch * high * heads * (per + 2) * dim <= 1 << 28:
            break
    return {"op": op, "batch": batch, "low": rng.choice([0, high // 2, high]), "high": high, "salt": salt,
            "part": rng.choice([0, 0, _spread(rng, 1, high)]), "q_heads": heads * per, "heads": heads, "dim": dim,
            "causal": rng.random() < 0.75, "type": kind, "pad": rng.choice([0, 8 * rng.randrange(1, 9), 2 * heads * dim])}


def _lengths(case):
    """How many tokens each sequence has: between low and high, the first one high."""
    rng = random.Random(case["salt"])
    return [case["high"]] + [rng.randint(case["low"], case["high"]) for _ in range(case["batch"] - 1)]


def _queries(case):
    """How many of a sequence's tokens are queries, the last ones."""
    if case["op"] == "qattn":
        return [case["tokens"]] * case["batch"]
    return [min(n, case["part"] or n) for n in _lengths(case)]


def _starts(counts):
    out = [0]
    for n in counts:
        out.append(out[-1] + n)
    return out


# ------------------------------------------------------------------ inputs
def _rows(g, tokens, heads, dim, pad, kind, scale=1.0):
    """[tokens][heads][dim] with `pad` elements between the tokens: normal, a few channels larger than the others."""
    x = torch.randn(tokens, heads * dim + pad, generator=g, device="cuda")
    x *= torch.where(torch.rand(heads * dim + pad, generator=g, device="cuda") < 0.01, 6.0, scale)
    return x.to(TYPES[kind])[:, :heads * dim].unflatten(1, (heads, dim))


def _table(positions, rot):
    """cos and sin of rot / 2 angles for each position, computed in 64 bits: [positions][rot]."""
    f = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)
    a = torch.arange(positions, dtype=torch.float64, device="cuda")[:, None] * f
    return torch.cat([a.cos(), a.sin()], 1).float()


def _head_bytes(case):
    return case["page"] * (case["dim"] + 4 * (case["dim"] // case["group"]))


def _pack(case, pages, codes, scales):
    """Fills pages [pages][heads][bytes] with codes [2][pages][page][heads][dim] and scales [2][...][dim / group]."""
    page, dim = case["page"], case["dim"]
    at, n, heads = page * dim // 2, codes.shape[1], codes.shape[3]
    codes = codes.transpose(2, 3)                                     # [2][pages][heads][page][dim]
    # keys: words of 8 channels, word w = 4 u + g at place g * dim / 32 + u; channels 2 j, 2 j + 1 in nibbles j, j + 4
    k = codes[0].unflatten(-1, (dim // 32, 4, 4, 2)).movedim(-1, -2).transpose(-3, -4).flatten(-4).unflatten(-1, (dim // 2, 2))
    pages[:, :, :at] = (k[..., 0] | k[..., 1] << 4).flatten(2)
    # values: channel 16 (4 h + n) + m in nibble n of the 16 bits [token / 4][m][h][token % 4]
    v = codes[1].reshape(n, heads, page // 4, 4, dim // 64, 2, 2, 16).permute(0, 1, 2, 7, 4, 3, 5, 6)
    pages[:, :, at:2 * at] = (v[..., 0] | v[..., 1] << 4).flatten(2)
    pages[:, :, 2 * at:] = scales.transpose(2, 3).permute(1, 2, 0, 3, 4).flatten(2).contiguous().view(torch.uint8)


def _unpack(case, pages):
    """(codes, scales) of pages, as _pack takes them, codes as int32."""
    page, dim = case["page"], case["dim"]
    at, n, heads = page * dim // 2, pages.shape[0], pages.shape[1]
    raw = pages.int()
    k = torch.stack([raw[:, :, :at] & 15, raw[:, :, :at] >> 4], -1).reshape(n, heads, page, 4, dim // 32, 2, 4)
    k = k.transpose(-3, -4).transpose(-1, -2).reshape(n, heads, page, dim)
    v = torch.stack([raw[:, :, at:2 * at] & 15, raw[:, :, at:2 * at] >> 4], -1).reshape(n, heads, page // 4, 16, dim // 64, 4, 4)
    v = v.permute(0, 1, 2, 5, 4, 6, 3).reshape(n, heads, page, dim)
    scales = pages[:, :, 2 * at:].contiguous().view(torch.bfloat16).reshape(n, heads, 2, page, dim // case["group"])
    return torch.stack([k, v]).transpose(2, 3), scales.permute(2, 0, 3, 1, 4)


def _quantise(case, x):
    """(codes, scales) of real numbers [..., dim] in fp32."""
    u = x.unflatten(-1, (-1, case["group"]))
    top, low = u.amax(-1, keepdim=True), u.amin(-1, keepdim=True)
    s = (torch.where(top >= -low, top, low) * -0.125).bfloat16()
    s = torch.where(s.abs() < LEAST, torch.zeros_like(s), s)
    r = torch.where(s == 0, torch.zeros_like(top), torch.div(torch.ones_like(top), s.float()))
    return ((u * r).round().clamp(-8, 7) + 8).to(torch.uint8).flatten(-2), s.squeeze(-1)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    op, kind, s = case["op"], case["type"], {"case": case}
    if op == "heads":
        tokens, dim, rot = case["tokens"], case["dim"], case["rot"]
        hq, hk = case["q_heads"], case["k_heads"]
        both = _rows(g, tokens, hq + hk, dim, case["pad"], kind)
        s["q"], s["k"] = both[:, :hq], both[:, hq:]
        s["wq"], s["wk"] = [(1 + 0.25 * torch.randn(dim, generator=g, device="cuda")).to(TYPES[kind]) if case["norm"] else None
                            for _ in range(2)]
        s["positions"] = 40000
        s["table"] = _table(s["positions"], rot)
        first = int(torch.randint(s["positions"] - tokens, (1,), generator=g, device="cuda"))
        s["position"] = torch.arange(first, first + tokens, dtype=torch.int32, device="cuda")
        s["yq"] = torch.empty(tokens, hq, dim, dtype=TYPES[kind], device="cuda")
        s["yk"] = torch.empty(tokens, hk, dim, dtype=TYPES[kind], device="cuda")
        return s
    heads, dim = case["heads"], case["dim"]
    if op == "attn":
        nk, nq = _starts(_lengths(case)), _starts(_queries(case))
        s["q"] = _rows(g, nq[-1], case["q_heads"], dim, case["pad"], kind)
        s["k"] = _rows(g, nk[-1], heads, dim, case["pad"], kind)
        s["v"] = _rows(g, nk[-1], heads, dim, case["pad"], kind)
        s["nq"], s["nk"] = nq, nk
        s["q_start"], s["k_start"] = [torch.tensor(a, dtype=torch.int32, device="cuda") for a in (nq, nk)]
        s["y"] = torch.empty(nq[-1], case["q_heads"], dim, dtype=TYPES[kind], device="cuda")
        s["workspace"] = torch.empty(WORKSPACE, dtype=torch.uint8, device="cuda")
        return s
    page = case["page"]
    if op == "cache":
        # runs of tokens of one sequence each, every one from the middle of a page on
        tokens, run = case["tokens"], case["run"]
        both = _rows(g, tokens, 2 * heads, dim, case["pad"], kind)
        s["k"], s["v"] = both[:, :heads], both[:, heads:]
        each = 2 + run // page
        runs = -(-tokens // run)
        s["pages"] = runs * each
        order = torch.randperm(s["pages"], generator=g, device="cuda").reshape(runs, each)
        t = torch.arange(tokens, device="cuda")
        at = t % run + torch.randint(page, (runs,), generator=g, device="cuda")[t // run]
        s["slots"] = (order[t // run, at // page] * page + at % page).int()
        s["cache"] = torch.zeros(s["pages"], heads, _head_bytes(case), dtype=torch.uint8, device="cuda")
        s["yk"], s["yv"] = [torch.empty(tokens, heads, dim, dtype=TYPES[kind], device="cuda") for _ in range(2)]
        return s
    # a sequence's pages lie anywhere in the cache
    lens = _lengths(case)
    used = [-(-n // page) for n in lens]
    s["pages"] = sum(used) + 3
    s["cache"] = torch.empty(s["pages"], heads, _head_bytes(case), dtype=torch.uint8, device="cuda")
    step = max(1, (1 << 25) // (2 * page * heads * dim))
    bias = 0.5 * torch.randn(2, 1, 1, heads, dim, generator=g, device="cuda")
    for a in range(0, s["pages"], step):
        part = s["cache"][a:a + step]
        x = torch.randn(2, len(part), page, heads, dim, generator=g, device="cuda")
        _pack(case, part, *_quantise(case, x + bias))
    order = torch.randperm(s["pages"], generator=g, device="cuda").int()
    s["ld_table"] = max(1, max(used))
    s["tables"] = torch.zeros(case["batch"], s["ld_table"], dtype=torch.int32, device="cuda")
    first = 0
    for b, n in enumerate(used):
        s["tables"][b, :n] = order[first:first + n]
        first += n
    s["lens"] = lens
    s["lengths"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    queries = case["batch"] * case["tokens"]
    s["q"] = _rows(g, queries, case["q_heads"], dim, 0, kind)
    s["nq"] = _starts(_queries(case))
    s["q_start"] = torch.tensor(s["nq"], dtype=torch.int32, device="cuda")
    s["y"] = torch.empty(queries, case["q_heads"], dim, dtype=TYPES[kind], device="cuda")
    s["workspace"] = torch.empty(WORKSPACE, dtype=torch.uint8, device="cuda")
    return s


# -------------------------------------------------------------- plain forms
def _plain_heads(case, x, weight, s):
    u, dim, rot = x.float(), case["dim"], case["rot"]
    if weight is not None:
        u = u / torch.sqrt((u * u).mean(-1, keepdim=True) + EPS) * weight.float()
    row = s["table"][s["position"].long()][:, None]
    c, n = row[..., :rot // 2], row[..., rot // 2:]
    if case["pairs"] == "halves":
        a, b = u[..., :rot // 2], u[..., rot // 2:rot]
        turned = torch.cat([a * c - b * n, b * c + a * n], -1)
    else:
        a, b = u[..., 0:rot:2], u[..., 1:rot:2]
        turned = torch.stack([a * c - b * n, b * c + a * n], -1).flatten(-2)
    return torch.cat([turned, u[..., rot:]], -1).to(TYPES[case["type"]])


def _plain_attention(q, k, v, causal, out):
    """One sequence: q [n][q_heads][dim], k and v [keys][heads][dim] in fp32, into out."""
    n, keys, dim = q.shape[0], k.shape[0], q.shape[2]
    if n == 0:
        return
    if keys == 0:
        out.zero_()
        return
    per = q.shape[1] // k.shape[1]
    row = torch.arange(n, device="cuda")[:, None] + (keys - n)
    hidden = (torch.arange(keys, device="cuda")[None, :] > row) if causal else None
    for h in range(k.shape[1]):
        kh, vh = k[:, h].t().contiguous(), v[:, h].contiguous()
        part = q[:, h * per:(h + 1) * per].reshape(n * per, dim)
        p = ((part @ kh) * dim ** -0.5).view(n, per, keys)
        if causal:
            p.masked_fill_(hidden[:, None], float("-inf"))
        p -= p.amax(2, keepdim=True).clamp_min(-3e38)
        p = p.exp_().view(n * per, keys)
        total = p.sum(1, keepdim=True)
        o = torch.where(total > 0, (p @ vh) / total.clamp_min(1e-38), 0.0)
        out[:, h * per:(h + 1) * per] = o.view(n, per, dim)


def _plain(s):
    case, op = s["case"], s["case"]["op"]
    if op == "heads":
        return {"q": _plain_heads(case, s["q"], s["wq"], s), "k": _plain_heads(case, s["k"], s["wk"], s)}
    if op == "cache":
        out = {}
        for name in ("k", "v"):
            codes, scales = _quantise(case, s[name].float())
            u = (codes.float() - 8).unflatten(-1, (-1, case["group"])) * scales.float().unsqueeze(-1)
            out[name] = u.flatten(-2).to(TYPES[case["type"]])
        return out
    y = torch.empty(s["y"].shape, device="cuda")
    for b in range(case["batch"]):
        q = s["q"][s["nq"][b]:s["nq"][b + 1]].float()
        if op == "attn":
            k, v = [s[name][s["nk"][b]:s["nk"][b + 1]].float() for name in ("k", "v")]
        else:
            n = s["lens"][b]
            used = -(-n // case["page"])
            codes, scales = _unpack(case, s["cache"][s["tables"][b, :used].long()])
            u = (codes.float() - 8).unflatten(-1, (-1, case["group"])) * scales.float().unsqueeze(-1)
            k, v = u.flatten(-2).flatten(1, 2)[:, :n]
        _plain_attention(q, k, v, case.get("causal", True), y[s["nq"][b]:s["nq"][b + 1]])
    return {"y": y.to(TYPES[case["type"]])}


def run(s):
    if not own:
        return _plain(s)
    from paper_2007_06919_amd import aqd
    case, op = s["case"], s["case"]["op"]
    kind = aqd.real_type(TYPES[case["type"]])
    if op == "heads":
        q, k, yq, yk = s["q"], s["k"], s["yq"], s["yk"]
        aqd.heads_run(case["tokens"], case["q_heads"], case["k_heads"], case["dim"], case["rot"],
                      aqd.PAIRS_HALVES if case["pairs"] == "halves" else aqd.PAIRS_NEIGHBOURS, kind, s["positions"], EPS,
                      q, q.stride(0), q.stride(1), k, k.stride(0), k.stride(1), s["wq"], s["wk"], s["position"], s["table"],
                      yq, yq.stride(0), yq.stride(1), yk, yk.stride(0), yk.stride(1))
        return {"q": yq, "k": yk}
    if op == "attn":
        q, k, v, y = s["q"], s["k"], s["v"], s["y"]
        aqd.attn_run(case["batch"], case["q_heads"], case["heads"], case["dim"], s["nq"][-1], s["nk"][-1], max(_queries(case)),
                     case["high"], case["causal"], kind, case["dim"] ** -0.5, q, q.stride(0), q.stride(1), k, k.stride(0), k.stride(1),
                     v, v.stride(0), v.stride(1), s["q_start"], s["k_start"], y, y.stride(0), y.stride(1), s["workspace"], WORKSPACE)
        return {"y": y}
    cache = aqd.QcacheDesc(case["heads"], case["dim"], case["group"], case["page"], s["pages"])
    if op == "cache":
        k, v, yk, yv = s["k"], s["v"], s["yk"], s["yv"]
        aqd.qcache_write(cache, case["tokens"], kind, k, k.stride(0), k.stride(1), v, v.stride(0), v.stride(1), s["slots"], s["cache"])
        aqd.qcache_read(cache, case["tokens"], kind, s["cache"], s["slots"], yk, yk.stride(0), yk.stride(1), yv, yv.stride(0), yv.stride(1))
        return {"k": yk, "v": yv}
    q, y = s["q"], s["y"]
    aqd.qattn_run(cache, case["batch"], case["q_heads"], s["nq"][-1], case["tokens"], case["high"], kind, case["dim"] ** -0.5,
                  q, q.stride(0), q.stride(1), s["q_start"] if case["tokens"] > 1 else None, s["cache"], s["tables"], s["ld_table"], s["lengths"],
                  y, y.stride(0), y.stride(1), s["workspace"], WORKSPACE)
    return {"y": y}


def _pairs(case):
    """How many keys all queries see together."""
    total = 0
    for n, keys in zip(_queries(case), _lengths(case)):
        if not case.get("causal", True):
            total += n * keys
        else:
            seen = min(n, keys)          # the last of the queries see any key
            total += seen * keys - seen * (seen - 1) // 2
    return total


def work(case):
    op, size = case["op"], SIZE[case["type"]]
    if op == "heads":
        tokens, n = case["tokens"], case["tokens"] * (case["q_heads"] + case["k_heads"]) * case["dim"]
        return {"bytes": 2 * n * size + tokens * (4 + 4 * case["rot"]) + (2 * case["dim"] * size if case["norm"] else 0), "flops": 8 * n}
    heads, dim = case["heads"], case["dim"]
    if op == "cache":
        n = 2 * case["tokens"] * heads
        packed = dim // 2 + 2 * (dim // case["group"])
        return {"bytes": 2 * n * (dim * size + packed) + 8 * case["tokens"], "flops": 6 * n * dim}
    queries = sum(_queries(case)) * case["q_heads"] * dim * size
    flops = 4 * dim * case["q_heads"] * _pairs(case)
    keys = sum(_lengths(case)) * heads
    if op == "attn":
        return {"bytes": 2 * queries + 2 * keys * dim * size, "flops": flops}
    return {"bytes": 2 * queries + keys * (dim + 4 * (dim // case["group"])), "flops": flops}


# ---------------------------------------------------------------- 64 bits
def _exact_values(case, s, b):
    """(keys, values) of sequence b in the cache, each [length][heads][dim], read code by code of its layout."""
    dim, page, n = case["dim"], case["page"], s["lens"][b]
    heads, at = case["heads"], case["page"] * case["dim"] // 2
    t, c = torch.arange(n, device="cuda"), torch.arange(dim, device="cuda")
    block = s["tables"][b].long()[t // page][:, None] * heads + torch.arange(heads, device="cuda")     # [n][heads]
    data, groups = s["cache"].view(-1), dim // case["group"]
    t, m, tile = (t % page)[:, None], c[None, :] % 16, c[None, :] // 16
    nibble = c % 8 // 2 + c % 2 * 4
    where_k = t * (dim // 2) + ((c // 8 % 4 * (dim // 32) + c // 32) * 4 + nibble // 2)[None, :]
    where_v = at + 2 * (((t // 4 * 16 + m) * (dim // 64) + tile // 4) * 4 + t % 4) + tile % 4 // 2
    out = []
    for side, (where, shift) in enumerate(((where_k, nibble % 2 * 4), (where_v, tile[0] % 2 * 4))):
        code = data[block[:, :, None] * _head_bytes(case) + where[:, None, :]].int() >> shift & 15
        row = (side * page + t) * groups + c[None, :] // case["group"]
        scale = data.view(torch.bfloat16)[(block[:, :, None] * _head_bytes(case) + 2 * at) // 2 + row[:, None, :]]
        out.append((code.to(torch.float64) - 8) * scale.to(torch.float64))
    return out


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op == "cache":
        # the scale is 16 bits wide by definition, so is the choice of the code that stands for an element
        out = {}
        for name in ("k", "v"):
            x = s[name].to(torch.float64).unflatten(2, (case["dim"] // case["group"], case["group"]))
            size = x.abs().amax(dim=3, keepdim=True)
            # positive where both signs reach the largest magnitude
            positive = (x == size).any(dim=3, keepdim=True)
            step = torch.where(positive, size, -size).div(-8).to(torch.bfloat16).to(torch.float64)
            steps = torch.where(step.abs() >= LEAST, torch.round(x / step), 0.0)
            out[name] = (torch.clamp(steps, min=-8, max=7) * step).flatten(2)
        return out
    if op == "heads":
        out, rot = {}, case["rot"]
        angle = s["table"].to(torch.float64)[s["position"].long()]
        z = torch.complex(angle[:, :rot // 2], angle[:, rot // 2:]).unsqueeze(1)
        for name in ("q", "k"):
            x = s[name].to(torch.float64)
            if case["norm"]:
                x = x * (x.pow(2).sum(2, keepdim=True) / case["dim"] + EPS).rsqrt() * s["w" + name].to(torch.float64)
            first = slice(0, rot // 2) if case["pairs"] == "halves" else slice(0, rot, 2)
            second = slice(rot // 2, rot) if case["pairs"] == "halves" else slice(1, rot, 2)
            w = torch.complex(x[..., first].contiguous(), x[..., second].contiguous()) * z
            x = x.clone()
            x[..., first], x[..., second] = w.real, w.imag
            out[name] = x
        return out
    y = torch.zeros(s["y"].shape, dtype=torch.float64, device="cuda")
    causal, per = case.get("causal", True), case["q_heads"] // case["heads"]
    for b in range(case["batch"]):
        q = s["q"][s["nq"][b]:s["nq"][b + 1]].to(torch.float64)
        if op == "attn":
            k, v = [s[name][s["nk"][b]:s["nk"][b + 1]].to(torch.float64) for name in ("k", "v")]
        else:
            k, v = _exact_values(case, s, b)
        n, keys = q.shape[0], k.shape[0]
        step = max(1, (1 << 27) // max(1, keys * per))
        for a in range(0, n, step):
            rows = q[a:a + step]
            see = min(keys, max(0, keys - n + a + len(rows))) if causal else keys
            if not see:
                continue
            last = torch.arange(a + keys - n, a + keys - n + len(rows), device="cuda")
            for h in range(case["heads"]):
                part = rows[:, h * per:(h + 1) * per].reshape(-1, case["dim"])
                logits = torch.mm(part, k[:see, h].t().contiguous()) / case["dim"] ** 0.5
                logits = logits.view(len(rows), per, see)
                if causal:
                    logits += torch.where(torch.arange(see, device="cuda")[None] <= last[:, None], 0.0, float("-inf"))[:, None].to(torch.float64)
                weight = torch.softmax(logits, 2).nan_to_num(0.0).view(-1, see)
                y[s["nq"][b] + a:s["nq"][b] + a + len(rows), h * per:(h + 1) * per] = torch.mm(weight, v[:see, h].contiguous()).view(len(rows), per, -1)
    return {"y": y}

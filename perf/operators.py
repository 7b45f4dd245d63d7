"""Performance cases of the 8-bit linear operators: rows of real numbers made into
8-bit codes with one scale per row (``qrows``), the same behind a residual's addition
and a root-mean-square norm (``qnorm``), and the matrix product of such codes with
8-bit weights that have one scale per output channel (``qlin``), plain or as the two
halves of a gated unit.

``run`` computes an operator in elementary torch operations in 32 bits, or, where
``own`` is true, by the library's entry points. The plain form's products are sums of
integers in fp32. Codes are int8 tensors: whole numbers beside their scales, equal to
the last one, because codes are made by one division per row and one product and one
rounding per element, in that order.
"""
from __future__ import annotations

import torch

own = False

TINY = 2.0 ** -119                 # smallest |row maximum| that a scale stands for
WORKSPACE = 64 << 20               # what a program keeps for the product's partial sums, one per stream
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}

MOST_FLOPS = 2 * 8192 ** 3         # the largest listed product
MOST_WEIGHTS = 2 * 16384 * 4096    # the largest listed weight matrix
MOST_NORM = 16384 * 4096           # the largest listed tensors of rows
MOST_ROWS = 8192 * 11000


def listed():
    return [
        # one token's hidden state in front of a block: what a call costs at least
        {"name": "norm_1x4096_bf16", "op": "qnorm", "rows": 1, "cols": 4096, "ld": 4096, "type": "bf16", "residual": True},
        # an odd number of fp32 channels, packed: no row but the first is aligned; the first norm, which has no residual
        {"name": "norm_301x2051_f32", "op": "qnorm", "rows": 301, "cols": 2051, "ld": 2051, "type": "f32", "residual": False},
        # a batch of prompts in front of a block
        {"name": "norm_16384x4096_bf16", "op": "qnorm", "rows": 16384, "cols": 4096, "ld": 4096, "type": "bf16", "residual": True},
        # the hidden units of a feed-forward block for 64 sequences that decode together
        {"name": "rows_64x16384_bf16", "op": "qrows", "rows": 64, "cols": 16384, "ld": 16384, "type": "bf16"},
        # the same for a batch of prompts, half precision, a slice of wider rows
        {"name": "rows_8192x11000_f16", "op": "qrows", "rows": 8192, "cols": 11000, "ld": 11016, "type": "f16"},
        # one token through a square projection
        {"name": "lin_1x4096x4096_bf16", "op": "qlin", "rows": 1, "n": 4096, "k": 4096, "ld": 4096, "type": "bf16",
         "bias": False, "gate": False},
        # 16 sequences that decode together, gated unit: every weight is read for a few rows
        {"name": "gate_16x16384x4096_bf16", "op": "qlin", "rows": 16, "n": 16384, "k": 4096, "ld": 4096, "type": "bf16",
         "bias": False, "gate": True},
        # odd everywhere, packed: rows of weights and codes start at any byte
        {"name": "lin_77x1003x515_f32", "op": "qlin", "rows": 77, "n": 1003, "k": 515, "ld": 515, "type": "f32",
         "bias": True, "gate": False},
        # a short prompt through the second layer of a feed-forward block: few tiles, a long sum
        {"name": "lin_192x4096x16384_bf16", "op": "qlin", "rows": 192, "n": 4096, "k": 16384, "ld": 16384, "type": "bf16",
         "bias": False, "gate": False},
        # the detectors' 720 class scores at the 22300 positions of the five levels of an 800 x 1333 image, as fp32
        {"name": "lin_22300x720x256_f32", "op": "qlin", "rows": 22300, "n": 720, "k": 256, "ld": 256, "type": "f32",
         "bias": True, "gate": False},
        # a long prompt through a gated unit
        {"name": "gate_2048x11264x4096_bf16", "op": "qlin", "rows": 2048, "n": 11264, "k": 4096, "ld": 4096, "type": "bf16",
         "bias": False, "gate": True},
        # a batch of prompts through a wide square projection
        {"name": "lin_8192x8192x8192_bf16", "op": "qlin", "rows": 8192, "n": 8192, "k": 8192, "ld": 8192, "type": "bf16",
         "bias": False, "gate": False},
    ]


def _spread(rng, low, high):
    """A size between low and high, even over its logarithm; a third of them any number, the others multiples of 16 to 256."""
    v = low * (high / low) ** rng.random()
    step = 1 if v < 32 else rng.choice([1, 16, 256 if v > 512 else 32])
    return max(low, min(high, int(round(v / step)) * step))


def draw(rng):
    op = rng.choice(["qnorm", "qrows", "qlin", "qlin", "qlin"])
    kind = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op != "qlin":
        most = (MOST_NORM if op == "qnorm" else MOST_ROWS) * 2 // SIZE[kind]
        while True:
            rows, cols = _spread(rng, 1, 16384), _spread(rng, 64, 16384)
            if rows * cols <= most:
                break
        ld = rng.choice([cols, cols, cols + 8, cols + rng.randrange(1, 64)])
        case = {"op": op, "rows": rows, "cols": cols, "ld": ld, "type": kind}
        return dict(case, residual=rng.random() < 0.75) if op == "qnorm" else case
    while True:
        rows, n, k = _spread(rng, 1, 16384), _spread(rng, 64, 16384), _spread(rng, 64, 16384)
        gate = rng.random() < 0.35
        wide = 2 * n if gate else n
        if 2 * rows * wide * k <= MOST_FLOPS and wide * k <= MOST_WEIGHTS and rows * max(n * SIZE[kind], k) <= 1 << 28:
            break
    # a program that chooses its own layout pads rows to 16 bytes; one that is handed a tensor may not be able to
    ld = k if k % 16 == 0 or rng.random() < 0.4 else -(-k // 16) * 16
    return {"op": op, "rows": rows, "n": n, "k": k, "ld": ld, "type": kind, "bias": rng.random() < 0.4, "gate": gate}


def _reals(g, rows, cols, ld, kind):
    """Activations: normal, a few channels much larger than the others, rows of unequal size, now and then a row of padding."""
    x = torch.randn(rows, ld, generator=g, device="cuda")
    x *= torch.where(torch.rand(ld, generator=g, device="cuda") < 0.004, 24.0, 1.0)
    x *= torch.exp2(2 * torch.rand(rows, 1, generator=g, device="cuda"))
    if rows >= 64:
        x[int(torch.randint(rows, (1,), generator=g, device="cuda"))] = 0
    return x.to(TYPES[kind])[:, :cols]


def _codes(g, rows, k, ld):
    """Signed 8-bit codes as quantised rows have them: normal, the largest near 127."""
    c = torch.empty(rows, ld, dtype=torch.int8, device="cuda")
    step = max(1, (1 << 26) // ld)
    for at in range(0, rows, step):
        part = torch.randn(min(step, rows - at), ld, generator=g, device="cuda")
        c[at:at + step] = (part * 34).round_().clamp_(-127, 127).to(torch.int8)
    return c[:, :k]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rows, s = case["rows"], {"case": case}
    if case["op"] == "qlin":
        n, k, wide = case["n"], case["k"], case["n"] * (2 if case["gate"] else 1)
        s["x"] = _codes(g, rows, k, case["ld"])
        s["w"] = _codes(g, wide, k, case["ld"])
        # scales that leave outputs of about 1
        s["x_scales"] = (0.5 + torch.rand(rows, generator=g, device="cuda")) / 34
        s["w_scales"] = (0.5 + torch.rand(wide, generator=g, device="cuda")) / (34 * k ** 0.5)
        s["bias"] = torch.randn(wide, generator=g, device="cuda") if case["bias"] else None
        s["y"] = torch.empty(rows, n, dtype=TYPES[case["type"]], device="cuda")
        s["workspace"] = torch.empty(WORKSPACE, dtype=torch.uint8, device="cuda")
        return s
    cols = case["cols"]
    s["x"] = _reals(g, rows, cols, case["ld"], case["type"])
    s["codes"] = torch.empty(rows, cols, dtype=torch.int8, device="cuda")
    s["scales"] = torch.empty(rows, device="cuda")
    if case["op"] == "qnorm":
        s["residual"] = _reals(g, rows, cols, cols, case["type"]) if case["residual"] else None
        s["sum"] = torch.empty(rows, cols, dtype=TYPES[case["type"]], device="cuda") if case["residual"] else None
        s["weight"] = (1 + 0.25 * torch.randn(cols, generator=g, device="cuda")).to(TYPES[case["type"]])
        s["eps"] = 1e-5
    return s


def _code(u):
    """(codes, row maximum) of rows u in fp32."""
    m = u.abs().amax(dim=1, keepdim=True).clamp_min(TINY)
    return (u * torch.div(torch.full_like(m, 127.0), m)).round().to(torch.int8), m


def _plain(s):
    case = s["case"]
    if case["op"] == "qlin":
        y = s["x"].float() @ s["w"].float().t()
        y = y * s["x_scales"][:, None] * s["w_scales"][None, :]
        if case["bias"]:
            y = y + s["bias"]
        if case["gate"]:
            gate, value = y[:, :case["n"]], y[:, case["n"]:]
            y = gate / (1 + torch.exp(-gate)) * value
        return {"y": y.to(TYPES[case["type"]])}
    u = s["x"].float()
    if case["op"] == "qrows":
        codes, m = _code(u)
        return {"codes": codes, "scales": (m / 127)[:, 0]}
    out = {}
    if case["residual"]:
        u = u + s["residual"].float()
        out["sum"] = u.to(TYPES[case["type"]])
    codes, m = _code(u * s["weight"].float())
    rms = torch.sqrt((u * u).mean(dim=1, keepdim=True) + s["eps"])
    return dict(out, codes=codes, scales=(m / rms / 127)[:, 0])


def run(s):
    if not own:
        return _plain(s)
    from paper_2007_06919_amd import aqd
    case, x = s["case"], s["x"]
    rows = case["rows"]
    if case["op"] == "qlin":
        y = s["y"]
        aqd.qlin_run(rows, case["n"], case["k"], aqd.real_type(y), aqd.QLIN_SILU_GATE if case["gate"] else aqd.QLIN_PLAIN,
                     x, x.stride(0), s["x_scales"], s["w"], s["w"].stride(0), s["w_scales"], s["bias"], y, y.stride(0),
                     s["workspace"], WORKSPACE)
        return {"y": y}
    cols, codes, scales = case["cols"], s["codes"], s["scales"]
    if case["op"] == "qrows":
        aqd.qrows_run(rows, cols, aqd.real_type(x), x, x.stride(0), codes, codes.stride(0), scales)
        return {"codes": codes, "scales": scales}
    r, total = s["residual"], s["sum"]
    aqd.qnorm_run(rows, cols, aqd.real_type(x), s["eps"], x, x.stride(0), r, cols, s["weight"], total, cols, codes,
                  codes.stride(0), scales)
    return {"codes": codes, "scales": scales} if r is None else {"sum": total, "codes": codes, "scales": scales}


def work(case):
    if case["op"] == "qlin":
        rows, n, k, wide = case["rows"], case["n"], case["k"], case["n"] * (2 if case["gate"] else 1)
        return {"bytes": (rows + wide) * (k + 4) + (4 * wide if case["bias"] else 0) + rows * n * SIZE[case["type"]],
                "flops": 2 * rows * wide * k}
    rows, cols, size = case["rows"], case["cols"], SIZE[case["type"]]
    if case["op"] == "qrows":
        return {"bytes": rows * cols * (size + 1) + 4 * rows, "flops": 3 * rows * cols}
    return {"bytes": rows * cols * (size * (3 if case["residual"] else 1) + 1) + 4 * rows + cols * size,
            "flops": 7 * rows * cols}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "qlin":
        x = s["x"].to(torch.float64) * s["x_scales"].to(torch.float64).unsqueeze(1)
        parts = []
        for half in range(2 if case["gate"] else 1):
            at = slice(half * case["n"], (half + 1) * case["n"])
            w = s["w"][at].to(torch.float64) * s["w_scales"][at].to(torch.float64).unsqueeze(1)
            part = torch.mm(x, w.t().contiguous())
            if s["bias"] is not None:
                part += s["bias"][at].to(torch.float64)
            parts.append(part)
        return {"y": parts[0] if len(parts) == 1 else parts[0] * torch.sigmoid(parts[0]) * parts[1]}
    t = s["x"].to(torch.float64)
    out = {}
    if case["op"] == "qnorm" and case["residual"]:
        t = t + s["residual"].to(torch.float64)
        out["sum"] = t
    if case["op"] == "qnorm":
        t = t * torch.rsqrt(t.pow(2).sum(1, keepdim=True) / case["cols"] + s["eps"]) * s["weight"].to(torch.float64)
    out["scales"] = t.abs().max(dim=1).values / 127
    # a code is a whole number: its rounding is the definition's, so 64 bits have no value of their own for it
    out["codes"] = None
    return out

"""Measured cases of microscaled 4-bit products, rotary positions and attention over packed prompts.

What one layer of a prompt encoder in reduced arithmetic runs, and what the linear layers of a denoising step would:

  quantize   a matrix to 4-bit codes (e2m1) with a scale for each group of columns of a row, and back to the values
             that they stand for (weights are transposed to [out, in] on the way): groups of 32 under a power of two, or groups of 16
             under an e4m3 scale and one power of two per row
  gemm       the product of two such operands
  rotary     rotation of channel pairs by angles that grow with the position, in packed sequences
  attend     softmax attention of packed sequences with grouped heads, every row over the keys up to its own

`own` chooses between the plain forms below (elementary torch operations) and the library's entry points.
"""
import math

import numpy as np
import torch

own = False

FLOOR = 2.0 ** -100          # the smallest magnitude that a group or row is scaled by
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)

TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"f16": 2, "bf16": 2, "f32": 4}


def listed():
    return [
        # the pooled state of one prompt before a product: a call that is nothing but latency
        {"name": "quantize_one_row", "op": "quantize", "rows": 1, "cols": 4096, "type": "bf16", "weight": False, "group": 16, "out": "bf16"},
        # GELU output of two packed 1024 x 1024 requests before the down-projection
        {"name": "quantize_mlp_rows", "op": "quantize", "rows": 9216, "cols": 12288, "type": "f16", "weight": False, "group": 16, "out": "f16"},
        # an up-projection as a checkpoint is loaded
        {"name": "quantize_weight", "op": "quantize", "rows": 4096, "cols": 12288, "type": "bf16", "weight": True, "group": 32, "out": "f32"},
        # a single row through a wide projection: the weights are read for it alone
        {"name": "gemm_one_row", "op": "gemm", "m": 1, "n": 18432, "k": 4096, "out": "f32", "bias": True, "group": 16},
        # a 77-token prompt through a ragged projection: no size a multiple of the tiles
        {"name": "gemm_ragged_prompt", "op": "gemm", "m": 77, "n": 1000, "k": 2056, "out": "bf16", "bias": True, "group": 32},
        # QKV projection of one 512 x 512 request with its text, or of a batch of prompts
        {"name": "gemm_qkv_512", "op": "gemm", "m": 1536, "n": 9216, "k": 4096, "out": "f16", "bias": True, "group": 16},
        # up-projection of one 2048 x 2048 request with its text
        {"name": "gemm_up_2048", "op": "gemm", "m": 16896, "n": 12288, "k": 4096, "out": "f16", "bias": True, "group": 16},
        # the new rows of four sequences, queries and keys in one call, half of each head rotated
        {"name": "rotary_single_rows", "op": "rotary", "lens": "1,1,1,1", "first": "16895,4607,1535,131071", "heads": 40, "dim": 128,
         "rotary": 64, "interleaved": True, "factor": 1.0, "ramp": "", "type": "bf16", "inverse": False},
        # a batch of prompts at several times the trained length
        {"name": "rotary_prompts", "op": "rotary", "lens": "16384,4097,2500,77", "first": "0,0,0,0", "heads": 40, "dim": 128,
         "rotary": 128, "interleaved": False, "factor": 8.0, "ramp": "1,4,8192", "type": "f16", "inverse": False},
        # single new rows against the stored keys of four sequences
        {"name": "attend_single_rows", "op": "attend", "q_lens": "1,1,1,1", "kv_lens": "32768,4608,1536,5000", "heads": 32, "kv_heads": 8,
         "dim": 128, "type": "bf16"},
        # a batch of short prompts of a small encoder
        {"name": "attend_short_prompts", "op": "attend", "q_lens": "77,256,5,333,120,77", "kv_lens": "77,256,5,333,120,77", "heads": 12,
         "kv_heads": 4, "dim": 64, "type": "f16"},
        # one long prompt
        {"name": "attend_long_prompt", "op": "attend", "q_lens": "8192", "kv_lens": "8192", "heads": 32, "kv_heads": 8, "dim": 128,
         "type": "bf16"},
    ]


def _between(rng, low, high):
    """Whole number of [low, high], spread over the logarithm."""
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(["quantize", "gemm", "rotary", "attend", "attend"])
    kind = rng.choice(["f16", "bf16"])
    if op == "quantize":
        weight = rng.random() < 0.3
        cols = _between(rng, 1, 16384)
        rows = _between(rng, 1, min(16896, 9216 * 12288 // cols if not weight else 4096 * 12288 // cols))
        kind, group = rng.choice(["bf16", "f16", "f32"]), rng.choice([16, 32])
        # (fp32 quotients at a border between two codes are rounded before they are decided: such a value is a step off, of which a
        # 32-bit comparison of all values says nothing)
        out = rng.choice(["bf16", "f16"] if kind == "f32" and group == 16 else ["bf16", "f16", "f32"])
        return {"op": op, "rows": rows, "cols": cols, "type": kind, "weight": weight, "group": group, "out": out}
    if op == "gemm":
        k, n = _between(rng, 16, 12288), _between(rng, 8, 18432)
        top = 16896 * 12288 * 4096 // (n * k)
        return {"op": op, "m": _between(rng, 1, max(1, min(16896, top))), "n": n, "k": k, "out": rng.choice(["f16", "bf16", "f32"]),
                "bias": rng.random() < 0.7, "group": rng.choice([16, 32])}
    dim = rng.choice([64, 128])
    if op == "rotary":
        n, heads = rng.randint(1, 6), rng.randint(1, 40)
        lens = [_between(rng, 1, 16384 // n) for _ in range(n)]
        if rng.random() < 0.25:
            lens = [1] * n
        dim = rng.choice([dim, 80, 96])
        rotary = rng.choice([dim, dim, dim // 2, 32])
        scaled = rng.random() < 0.5
        return {"op": op, "lens": ",".join(map(str, lens)), "first": ",".join(str(rng.choice([0, _between(rng, 1, 200000)])) for _ in lens),
                "heads": heads, "dim": dim, "rotary": rotary, "interleaved": rng.random() < 0.5,
                "factor": rng.choice([2.0, 8.0, 40.0]) if scaled else 1.0, "ramp": rng.choice(["", "1,4,8192", "1,32,4096"]) if scaled else "",
                "type": rng.choice(["f16", "bf16", "f32"]), "inverse": rng.random() < 0.2}
    kv_heads = rng.choice([1, 2, 3, 4, 8])
    heads = kv_heads * rng.randint(1, (32 if dim == 128 else 24) // kv_heads)
    n = rng.randint(1, 6)
    if rng.random() < 0.4:                                           # a few new rows, each against a longer context
        kv = [_between(rng, 1, 32768 // n) for _ in range(n)]
        q = [min(l, rng.choice([1, 1, 1, 2, 5])) for l in kv]
    else:
        q = [_between(rng, 1, int(8192 / math.sqrt(n))) for _ in range(n)]
        # whole prompts, or the rest of prompts whose beginning is stored
        kv = q if rng.random() < 0.7 else [min(int(8192 / math.sqrt(n)), l + _between(rng, 1, 1000)) for l in q]
    return {"op": op, "q_lens": ",".join(map(str, q)), "kv_lens": ",".join(map(str, kv)), "heads": heads, "kv_heads": kv_heads, "dim": dim,
            "type": kind}


def _whole(text):
    return [int(x) for x in text.split(",")]


def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32)


def _operand(gen, rows, k, group, level):
    """A quantised operand that a caller has in hand: codes [rows, ceil(k / 2)] two to a byte (rows 16-byte aligned), scale bytes in tiles of
    128 rows x 4 groups, fp32 row scales."""
    pitch = (k + 31) // 32 * 16
    edges = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device="cuda")
    value = 2.5 * _normal(gen, rows, 2 * pitch)
    code = torch.bucketize(value.abs(), edges).to(torch.uint8) + 8 * (value < 0).to(torch.uint8)
    code[:, k:] = 0
    codes = (code[:, 0::2] + 16 * code[:, 1::2])[:, :(k + 1) // 2]
    tiles, chunks = (rows + 127) // 128, (k + 4 * group - 1) // (4 * group)
    if group == 16:
        scales = (64.0 * torch.exp(0.5 * _normal(gen, tiles, chunks, 512))).clamp(max=448.0).to(torch.float8_e4m3fn).view(torch.uint8)
        row_scales = level / 64.0 * torch.exp(0.5 * _normal(gen, rows))
    else:
        scales = (127.0 + math.log2(level) + _normal(gen, tiles, chunks, 512)).round().to(torch.uint8)
        row_scales = None
    return codes, scales, row_scales


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    state = {"case": case}
    if case["op"] == "quantize":
        x = _normal(gen, case["rows"], case["cols"])
        if case["weight"]:
            x *= 0.02
        else:
            x = torch.where(x > 0, x, 0.05 * x)                       # one-sided, as after a gated unit
            loud = torch.rand(case["cols"], generator=gen, device="cuda") < 0.004
            x = torch.where(loud, 20.0 * x, x)                        # a few loud channels
        state["x"] = x.to(TYPES[case["type"]])
    elif case["op"] == "gemm":
        state["a"], state["a_scales"], state["a_rows"] = _operand(gen, case["m"], case["k"], case["group"], 0.4)
        state["b"], state["b_scales"], state["b_rows"] = _operand(gen, case["n"], case["k"], case["group"], 0.01)
        state["bias"] = 0.1 * _normal(gen, case["n"]) if case["bias"] else None
    elif case["op"] == "rotary":
        lens, first = _whole(case["lens"]), _whole(case["first"])
        width = case["heads"] * case["dim"]
        # queries and keys are the first columns of the buffer that a projection wrote; the values behind them stay
        state["x"] = _normal(gen, sum(lens), width + 8 * case["dim"]).to(TYPES[case["type"]])[:, :width]
        state["lens"], state["first"] = lens, first
        state["ramp"] = tuple(_whole(case["ramp"])) if case["ramp"] else None
    else:
        q_lens, kv_lens = _whole(case["q_lens"]), _whole(case["kv_lens"])
        width, kv_width = case["heads"] * case["dim"], case["kv_heads"] * case["dim"]
        kind = TYPES[case["type"]]
        if q_lens == kv_lens:
            qkv = _normal(gen, sum(q_lens), width + 2 * kv_width)     # one packed buffer [rows, q | k | v]
            qkv[:, :width] *= 1.5
            qkv = qkv.to(kind)
            state["q"], state["k"], state["v"] = qkv[:, :width], qkv[:, width:width + kv_width], qkv[:, width + kv_width:]
        else:
            state["q"] = (1.5 * _normal(gen, sum(q_lens), width)).to(kind)
            state["k"], state["v"] = (_normal(gen, sum(kv_lens), kv_width).to(kind) for _ in range(2))
        state["q_lens"], state["kv_lens"] = q_lens, kv_lens
    return state


# --------------------------------------------------------------------------------------------- plain forms
def _nearest_level(x):
    """|x| <= 6 to the nearest value of the format, ties to the even code."""
    a = x.abs()
    step = torch.where(a < 2.0, 0.5, torch.where(a < 4.0, 1.0, 2.0))
    return torch.copysign(torch.round(a / step) * step, x)            # (torch.round takes ties to even)


def _plain_quantize(state):
    case = state["case"]
    x, group = state["x"].float(), case["group"]
    if case["weight"]:
        x = x.t()
    rows, cols = x.shape
    parts = torch.nn.functional.pad(x, (0, -cols % group)).reshape(rows, -1, group)
    top = parts.abs().amax(dim=2, keepdim=True)
    power = lambda e: ((e + 127) << 23).int().view(torch.float32)     # 2^e, whose bits are its exponent
    if group == 32:
        mantissa, exponent = torch.frexp(top.clamp(min=FLOOR))        # top = mantissa * 2^exponent, mantissa in [1/2, 1)
        exponent = exponent - torch.where(mantissa <= 0.75, 3, 2)     # the smallest with top <= 6 * 2^exponent
        values = _nearest_level((parts * power(-exponent)).clamp(-6.0, 6.0)) * power(exponent)
        row_scales = None
    else:
        mantissa, exponent = torch.frexp(x.abs().amax(dim=1).clamp(min=FLOOR)[:, None, None])
        exponent = exponent - torch.where(mantissa <= 0.65625, 12, 11)            # the smallest with row top <= 6 * 448 * 2^exponent
        scale = ((top * power(-exponent)) / 6.0).clamp(max=448.0).to(torch.float8_e4m3fn).float()
        code = torch.where(scale > 0, (parts * power(-exponent)) / torch.where(scale > 0, scale, 1.0), 0.0)
        values = _nearest_level(code.clamp(-6.0, 6.0)) * scale * power(exponent)
        row_scales = power(exponent)[:, 0, 0]
    return {"values": values.reshape(rows, -1)[:, :cols].to(TYPES[case["out"]]), "row_scales": row_scales}


def _plain_operand(codes, scales, row_scales, k, group):
    """fp32 [rows, k] that an operand stands for."""
    levels = torch.tensor(LEVELS + tuple(-v for v in LEVELS), device="cuda")
    rows = codes.shape[0]
    value = torch.stack([levels[(codes & 15).int()], levels[(codes >> 4).int()]], dim=2).reshape(rows, -1)[:, :k]
    # a tile's bytes: row % 32, row / 32, group
    scale = scales.view(torch.float8_e4m3fn).float() if group == 16 else torch.exp2(scales.float() - 127.0)
    tiles, chunks = scale.shape[:2]
    scale = scale.reshape(tiles, chunks, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(tiles * 128, chunks * 4)[:rows]
    value = value * scale.repeat_interleave(group, dim=1)[:, :k]
    return value if row_scales is None else value * row_scales[:, None]


def _plain_gemm(state):
    case = state["case"]
    a = _plain_operand(state["a"], state["a_scales"], state["a_rows"], case["k"], case["group"])
    b = _plain_operand(state["b"], state["b_scales"], state["b_rows"], case["k"], case["group"])
    c = a @ b.t()
    if state["bias"] is not None:
        c = c + state["bias"]
    return c.to(TYPES[case["out"]])


def _places(lens, first):
    """Position of every packed row, in 64 bits."""
    starts = np.repeat(np.cumsum([0] + lens[:-1]), lens)
    return torch.from_numpy(np.arange(sum(lens)) - starts + np.repeat(first, lens)).cuda().double()


def _plain_rotary(state):
    case = state["case"]
    heads, dim, rotary = case["heads"], case["dim"], case["rotary"]
    freq = 10000.0 ** (-torch.arange(0, rotary, 2, device="cuda", dtype=torch.float64) / rotary)
    if state["ramp"] is None:
        freq = freq / case["factor"]
    else:
        low, high, trained = state["ramp"]
        keep = ((trained * freq / (2 * math.pi) - low) / (high - low)).clamp(0.0, 1.0)
        freq = freq * (keep + (1.0 - keep) / case["factor"])
    angle = _places(state["lens"], state["first"])[:, None] * freq
    cos, sin = torch.cos(angle).float()[:, None, :], torch.sin(angle).float()[:, None, :]
    if case["inverse"]:
        sin = -sin
    x = state["x"].float().reshape(-1, heads, dim)
    if case["interleaved"]:
        a, b = x[:, :, 0:rotary:2], x[:, :, 1:rotary:2]
        turned = torch.stack([a * cos - b * sin, a * sin + b * cos], dim=3).flatten(2)
    else:
        a, b = x[:, :, :rotary // 2], x[:, :, rotary // 2:rotary]
        turned = torch.cat([a * cos - b * sin, a * sin + b * cos], dim=2)
    return torch.cat([turned, x[:, :, rotary:]], dim=2).reshape(-1, heads * dim).to(TYPES[case["type"]])


def _padded(x, lens, heads):
    """fp32 [requests, heads, longest, dim], zeros behind a request's last row, and which rows exist."""
    local = np.arange(max(lens))[None, :]
    there = local < np.asarray(lens)[:, None]
    rows = torch.from_numpy(np.where(there, np.cumsum([0] + lens[:-1])[:, None] + local, 0)).cuda()
    there = torch.from_numpy(there).cuda()
    out = x[rows].float() * there[:, :, None]
    return out.reshape(len(lens), max(lens), heads, -1).transpose(1, 2), there


def _plain_attend(state):
    case = state["case"]
    heads, kv_heads, dim = case["heads"], case["kv_heads"], case["dim"]
    q, q_there = _padded(state["q"], state["q_lens"], heads)
    k, k_there = _padded(state["k"], state["kv_lens"], kv_heads)
    v, _ = _padded(state["v"], state["kv_lens"], kv_heads)
    scores = (q / math.sqrt(dim)) @ k.repeat_interleave(heads // kv_heads, dim=1).transpose(2, 3)
    before = torch.tensor(state["kv_lens"], device="cuda") - torch.tensor(state["q_lens"], device="cuda")
    last = before[:, None] + torch.arange(q.shape[2], device="cuda")[None, :]             # the last key that a row sees
    seen = (torch.arange(k.shape[2], device="cuda") <= last[:, :, None]) & k_there[:, None, :]
    scores.masked_fill_(~seen[:, None], -math.inf)
    top = scores.amax(3, keepdim=True)
    scores.sub_(torch.where(top > -math.inf, top, 0.0)).exp_()
    total = scores.sum(3, keepdim=True)
    out = (scores @ v.repeat_interleave(heads // kv_heads, dim=1)) / torch.where(total > 0, total, 1.0)
    return out.transpose(1, 2).flatten(2)[q_there].to(TYPES[case["type"]])


# --------------------------------------------------------------------------------------------- one pass
def run(state):
    case = state["case"]
    if own:
        from paper_2510_01565_b200 import binding as B
        if case["op"] == "quantize":
            quantize = B.dit_quantize_weight_fp4 if case["weight"] else B.dit_quantize_fp4
            codes, scales, row_scales = quantize(state["x"], case["group"])
            cols = case["rows"] if case["weight"] else case["cols"]
            return {"values": B.dit_dequantize_fp4(codes, scales, cols, case["group"], row_scales, out_dtype=TYPES[case["out"]]),
                    "row_scales": row_scales}
        if case["op"] == "gemm":
            return B.dit_gemm_fp4(state["a"], state["a_scales"], state["b"], state["b_scales"], case["k"], case["group"],
                                  a_row_scales=state["a_rows"], b_row_scales=state["b_rows"], bias=state["bias"], out_dtype=TYPES[case["out"]])
        if case["op"] == "rotary":
            return B.dit_rotary(state["x"], case["heads"], state["lens"], first=state["first"], rotary_dim=case["rotary"],
                                interleaved=case["interleaved"], factor=case["factor"], ramp=state["ramp"], inverse=case["inverse"])
        return B.dit_prompt_attention(state["q"], state["k"], state["v"], state["q_lens"], state["kv_lens"], case["heads"], case["kv_heads"])
    return {"quantize": _plain_quantize, "gemm": _plain_gemm, "rotary": _plain_rotary, "attend": _plain_attend}[case["op"]](state)


def work(case):
    if case["op"] == "quantize":
        rows, cols = (case["cols"], case["rows"]) if case["weight"] else (case["rows"], case["cols"])
        n, groups = rows * cols, rows * ((cols + case["group"] - 1) // case["group"])
        packed = rows * ((cols + 1) // 2) + groups + (4 * rows if case["group"] == 16 else 0)
        return {"bytes": n * (SIZE[case["type"]] + SIZE[case["out"]]) + 2 * packed, "flops": 5 * n}
    if case["op"] == "gemm":
        m, n, k = case["m"], case["n"], case["k"]
        each = (k + 1) // 2 + (k + case["group"] - 1) // case["group"] + (4 if case["group"] == 16 else 0)
        return {"bytes": (m + n) * each + (4 * n if case["bias"] else 0) + m * n * SIZE[case["out"]], "flops": 2 * m * n * k}
    if case["op"] == "rotary":
        n = sum(_whole(case["lens"])) * case["heads"]
        return {"bytes": 2 * n * case["dim"] * SIZE[case["type"]], "flops": 3 * n * case["rotary"]}
    q_lens, kv_lens = _whole(case["q_lens"]), _whole(case["kv_lens"])
    width, kv_width = case["heads"] * case["dim"], case["kv_heads"] * case["dim"]
    seen = sum(q * (kv - q) + q * (q + 1) // 2 for q, kv in zip(q_lens, kv_lens))         # (no request has more new rows than keys)
    return {"bytes": SIZE[case["type"]] * (2 * width * sum(q_lens) + 2 * kv_width * sum(kv_lens)), "flops": 4 * width * seen}


# --------------------------------------------------------------------------------------------- the definitions, in 64 bits
def _exact_operand(codes, scales, row_scales, k, group):
    rows = codes.shape[0]
    col, row = torch.arange(k, device="cuda"), torch.arange(rows, device="cuda")[:, None]
    code = (codes.int()[:, col // 2] >> (4 * (col % 2))) & 15
    exponent, mantissa = (code & 7) >> 1, (code & 1).double()
    value = torch.where(exponent > 0, (1.0 + 0.5 * mantissa) * torch.exp2(exponent.double() - 1.0), 0.5 * mantissa)
    value = torch.where(code >= 8, -value, value)
    g = col // group
    byte = scales[row // 128, g // 4, row % 32 * 16 + row % 128 // 32 * 4 + g % 4].int()
    if group == 32:
        return value * torch.exp2(byte.double() - 127.0)
    exponent, mantissa = byte >> 3, (byte & 7).double()
    scale = torch.where(exponent > 0, (1.0 + mantissa / 8) * torch.exp2(exponent.double() - 7.0), mantissa * 2.0 ** -9)
    return value * scale * row_scales.double()[:, None]


def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] == "quantize":
        x, group = state["x"].double(), case["group"]
        if case["weight"]:
            x = x.t()
        rows, cols = x.shape
        out, row_scales = torch.empty(rows, cols, device="cuda", dtype=torch.float64), None
        wide = (cols + group - 1) // group
        where = torch.arange(cols, device="cuda") // group
        top = torch.zeros(rows, wide, device="cuda", dtype=torch.float64).scatter_reduce_(1, where.expand(rows, cols), x.abs(), "amax")
        if group == 32:
            scale = torch.exp2(torch.round(torch.log2(top.clamp(min=FLOOR))) - 4.0)        # at least a step too small
            for _ in range(3):
                scale = torch.where(6.0 * scale < top.clamp(min=FLOOR), 2.0 * scale, scale)
        else:
            row_top = top.amax(1, keepdim=True).clamp(min=FLOOR)
            unit = torch.exp2(torch.round(torch.log2(row_top)) - 13.0)
            for _ in range(3):
                unit = torch.where(2688.0 * unit < row_top, 2.0 * unit, unit)
            row_scales = unit[:, 0]
            want = top / unit / 6.0
            step = 2.0 ** -9 * torch.ones_like(want)                   # e4m3: three bits behind the leading one
            for e in range(-5, 9):
                step = torch.where(want >= 2.0 ** e, 2.0 ** (e - 3), step)
            scale = torch.round(want / step) * step * unit
        levels = torch.tensor(LEVELS, device="cuda", dtype=torch.float64)
        for r in range(0, rows, 1024):                                 # the nearest level by its distance; of two, the even code
            s = scale[r:r + 1024, where]
            y = torch.where(s > 0, x[r:r + 1024].abs() / s.clamp(min=1e-300), 0.0).clamp(max=6.0)
            low = torch.bucketize(y, levels, right=True) - 1
            high = (low + 1).clamp(max=7)
            down, up = y - levels[low], levels[high] - y
            code = torch.where((up < down) | ((up == down) & (low % 2 == 1)), high, low)
            out[r:r + 1024] = torch.copysign(levels[code], x[r:r + 1024]) * s
        return {"values": out, "row_scales": row_scales}
    if case["op"] == "gemm":
        a = _exact_operand(state["a"], state["a_scales"], state["a_rows"], case["k"], case["group"])
        b = _exact_operand(state["b"], state["b_scales"], state["b_rows"], case["k"], case["group"])
        out = a @ b.t()
        return out if state["bias"] is None else out + state["bias"].double()
    if case["op"] == "rotary":
        heads, dim, rotary = case["heads"], case["dim"], case["rotary"]
        position = torch.cat([torch.arange(f, f + l, dtype=torch.float64) for f, l in zip(state["first"], state["lens"])]).cuda()
        out = state["x"].double().reshape(-1, heads, dim).clone()
        for i in range(rotary // 2):
            f = 10000.0 ** (-2.0 * i / rotary)
            share = 0.0
            if state["ramp"] is not None:
                low, high, trained = state["ramp"]
                share = min(1.0, max(0.0, (trained * f / (2.0 * math.pi) - low) / (high - low)))
            f = share * f + (1.0 - share) * f / case["factor"]
            turn = torch.polar(torch.ones_like(position), position * (-f if case["inverse"] else f))[:, None]
            i0, i1 = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + rotary // 2)
            z = torch.complex(out[:, :, i0], out[:, :, i1]) * turn
            out[:, :, i0], out[:, :, i1] = z.real, z.imag
        return out.reshape(-1, heads * dim)
    heads, kv_heads, dim = case["heads"], case["kv_heads"], case["dim"]
    out = torch.zeros(state["q"].shape, device="cuda", dtype=torch.float64)
    q0 = k0 = 0
    for lq, lk in zip(state["q_lens"], state["kv_lens"]):             # request by request, head by head
        for h in range(heads):
            g = h // (heads // kv_heads)
            q = state["q"][q0:q0 + lq, h * dim:(h + 1) * dim].double()
            k, v = (state[n][k0:k0 + lk, g * dim:(g + 1) * dim].double() for n in ("k", "v"))
            s = q @ k.t() / dim ** 0.5 + torch.full((lq, lk), -math.inf, device="cuda", dtype=torch.float64).triu(lk - lq + 1)
            out[q0:q0 + lq, h * dim:(h + 1) * dim] = torch.softmax(s, dim=1) @ v
        q0, k0 = q0 + lq, k0 + lk
    return out

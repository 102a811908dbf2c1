"""Measured cases of the block-scaled e4m3 product and of attention over selected key blocks.

Four operators, as a denoising step in reduced arithmetic uses them:

  quantize   a matrix to e4m3 codes with one scale for each 128 columns of a row (activations), or for each
             128 x 128 block (weights, which are transposed to [out, in] on the way)
  gemm       the product of two such operands, each block's partial sum scaled in 32 bits
  select     for every block of 128 query rows of a head, the key blocks with the largest product of the two
             blocks' mean rows (ties to the lowest block), the blocks of a request's last rows always among them
  attend     softmax attention of every query block over its selected key blocks only

`own` chooses between the plain forms below (elementary torch operations) and the library's entry points.
"""
import math

import numpy as np
import torch

own = False

BLOCK = 128
E4M3_MAX = 448.0
FLOOR = 2.0 ** -100          # the smallest magnitude a block is scaled by

TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"f16": 2, "bf16": 2, "f32": 4}


def listed():
    return [
        # one request's conditioning vector before a modulation product: a call that is nothing but latency
        {"name": "quantize_one_row", "op": "quantize", "rows": 1, "cols": 3072, "type": "bf16", "weight": False},
        # GELU output of two packed 1024 x 1024 requests before the down-projection
        {"name": "quantize_mlp_rows", "op": "quantize", "rows": 9216, "cols": 12288, "type": "f16", "weight": False},
        # an up-projection as a checkpoint is loaded
        {"name": "quantize_weight", "op": "quantize", "rows": 3072, "cols": 12288, "type": "bf16", "weight": True},
        # adaLN modulation of one request: the weights are read for a single row
        {"name": "gemm_one_row", "op": "gemm", "m": 1, "n": 18432, "k": 3072, "out": "f32", "bias": True},
        # a 77-token prompt through a ragged projection: no size a multiple of the blocks
        {"name": "gemm_ragged_prompt", "op": "gemm", "m": 77, "n": 1000, "k": 2056, "out": "bf16", "bias": True},
        # QKV projection of one 512 x 512 request with its text
        {"name": "gemm_qkv_512", "op": "gemm", "m": 1536, "n": 9216, "k": 3072, "out": "f16", "bias": True},
        # up-projection of one 2048 x 2048 request with its text
        {"name": "gemm_up_2048", "op": "gemm", "m": 16896, "n": 12288, "k": 3072, "out": "f16", "bias": True},
        # three small requests of the small model
        {"name": "select_small", "op": "select", "q_lens": "256,333,77", "kv_lens": "256,333,77", "heads": 6, "dim": 64,
         "keep": 2, "tail": 0, "type": "f16"},
        # one 2048 x 2048 request, a tenth of its key blocks kept, the 512 text rows always
        {"name": "select_2048", "op": "select", "q_lens": "16896", "kv_lens": "16896", "heads": 24, "dim": 128, "keep": 14,
         "tail": 512, "type": "f16"},
        # single new rows against the stored keys of four long requests
        {"name": "attend_one_row", "op": "attend", "q_lens": "1,1,1,1", "kv_lens": "16896,4608,1536,5000", "heads": 24, "dim": 128,
         "keep": 16, "tail": 0, "type": "f16"},
        # two 1024 x 1024 requests with text, a quarter of the blocks
        {"name": "attend_1024x2", "op": "attend", "q_lens": "4608,4608", "kv_lens": "4608,4608", "heads": 24, "dim": 128, "keep": 9,
         "tail": 512, "type": "bf16"},
        # one 2048 x 2048 request, a tenth of the blocks
        {"name": "attend_2048", "op": "attend", "q_lens": "16896", "kv_lens": "16896", "heads": 24, "dim": 128, "keep": 14,
         "tail": 512, "type": "f16"},
    ]


def _between(rng, low, high):
    """Whole number of [low, high], spread over the logarithm."""
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(["quantize", "gemm", "select", "attend"])
    if op == "quantize":
        weight = rng.random() < 0.3
        cols = _between(rng, 1, 15360)
        rows = _between(rng, 1, min(16896, 9216 * 12288 // cols if not weight else 3072 * 12288 // cols))
        return {"op": op, "rows": rows, "cols": cols, "type": rng.choice(["bf16", "f16"] if weight else ["f16", "bf16", "f32"]),
                "weight": weight}
    if op == "gemm":
        k, n = _between(rng, 16, 12288), _between(rng, 8, 18432)
        top = 16896 * 12288 * 3072 // (n * k)
        return {"op": op, "m": _between(rng, 1, max(1, min(16896, top))), "n": n, "k": k, "out": rng.choice(["f16", "bf16", "f32"]),
                "bias": rng.random() < 0.7}
    dim = rng.choice([64, 128])
    heads = rng.randint(4 if op == "select" else 1, 24 if dim == 128 else 16)
    n = rng.randint(1, 6)
    kv = [_between(rng, 1, 16896 // n) for _ in range(n)]
    if op == "select":
        kv[0] = _between(rng, 1000, 16896 // n)                       # one request at least that has a choice to make
    # a request's own rows attend to it, or a few new rows read a longer stored context
    q = kv if rng.random() < 0.7 else [_between(rng, 1, min(300, l)) for l in kv]
    blocks = max((l + BLOCK - 1) // BLOCK for l in kv)
    keep = rng.randint(1, max(1, min(14, blocks - 1)))
    tail = rng.choice([t for t in (0, 0, 77, 512) if t == 0 or t // BLOCK + 2 < keep])
    return {"op": op, "q_lens": ",".join(map(str, q)), "kv_lens": ",".join(map(str, kv)), "heads": heads, "dim": dim, "keep": keep,
            "tail": tail, "type": rng.choice(["f16", "bf16"])}


def _lens(text):
    return [int(x) for x in text.split(",")]


def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32)


def _rows_like(gen, lens, width):
    """Rows whose neighbourhoods resemble one another, as tokens of an image do: a slowly wandering mean per block
    of rows plus noise."""
    total = sum(lens)
    blocks = total // BLOCK + 2
    steps = _normal(gen, blocks, width)
    # a random walk that forgets: mean[i] = 0.8 mean[i - 1] + 0.6 step[i], as one product
    i = torch.arange(blocks, device="cuda", dtype=torch.float32)
    decay = torch.where(i[:, None] >= i[None, :], 0.8 ** (i[:, None] - i[None, :]).clamp(min=0), torch.zeros((), device="cuda"))
    mean = 0.6 * (decay @ steps)
    return 0.6 * mean[torch.arange(total, device="cuda") // BLOCK] + 0.8 * _normal(gen, total, width)


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
        return state
    if case["op"] == "gemm":
        m, n, k = case["m"], case["n"], case["k"]
        # operands a caller quantised before: codes [rows, pitch], of which the first k columns hold the operand
        pitch = (k + 15) // 16 * 16
        kb, nb = (k + BLOCK - 1) // BLOCK, (n + BLOCK - 1) // BLOCK
        state["a"] = (_normal(gen, m, pitch) * 120.0).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)[:, :k]
        state["b"] = (_normal(gen, n, pitch) * 120.0).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)[:, :k]
        state["a_scale"] = torch.exp(0.5 * _normal(gen, kb, m)) / 120.0
        state["b_scale"] = torch.exp(0.3 * _normal(gen, nb, kb)) * (0.02 / 120.0)
        state["bias"] = 0.1 * _normal(gen, n) if case["bias"] else None
        return state
    q_lens, kv_lens, width = _lens(case["q_lens"]), _lens(case["kv_lens"]), case["heads"] * case["dim"]
    kind = TYPES[case["type"]]
    if q_lens == kv_lens:
        # one packed buffer [rows, q | k | v], as a projection writes it
        state["qkv"] = torch.cat([_rows_like(gen, q_lens, width) for _ in range(3)], dim=1).to(kind)
        state["q"], state["k"], state["v"] = (state["qkv"][:, i * width:(i + 1) * width] for i in range(3))
    else:
        state["q"] = _rows_like(gen, q_lens, width).to(kind)
        state["k"], state["v"] = (_rows_like(gen, kv_lens, width).to(kind) for _ in range(2))
    state["q_lens"], state["kv_lens"] = q_lens, kv_lens
    state["keep"] = [case["keep"]] * len(q_lens)
    state["tail"] = [case["tail"]] * len(q_lens)
    if case["op"] == "attend":
        state["index"], state["count"] = _plain_select(state)
    return state


# --------------------------------------------------------------------------------------------- plain forms
def _plain_quantize(state):
    x, weight = state["x"].float(), state["case"]["weight"]
    if weight:
        x = x.t()
    rows, cols = x.shape
    x = torch.nn.functional.pad(x, (0, -cols % BLOCK, 0, -rows % BLOCK if weight else 0))
    tall = BLOCK if weight else 1
    blocks = x.reshape(x.shape[0] // tall, tall, x.shape[1] // BLOCK, BLOCK)
    top = blocks.abs().amax(dim=(1, 3), keepdim=True).clamp(min=FLOOR)
    codes = (blocks * (E4M3_MAX / top)).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
    scales = (top / E4M3_MAX)[:, 0, :, 0]
    return {"codes": codes.reshape(x.shape)[:rows, :cols], "scales": scales if weight else scales.t()}


def _plain_gemm(state):
    case = state["case"]
    n, k = case["n"], case["k"]
    a = state["a"].float() * state["a_scale"].repeat_interleave(BLOCK, dim=0)[:k].t()
    b = state["b"].float() * state["b_scale"].repeat_interleave(BLOCK, dim=0)[:n].repeat_interleave(BLOCK, dim=1)[:, :k]
    c = a @ b.t()
    if state["bias"] is not None:
        c = c + state["bias"]
    return c.to(TYPES[case["out"]])


def _grid(lens):
    """Blocks of a packed batch, request after request: rows [blocks, 128], which of them exist, the request of each
    block, its place in the request, and each request's first block."""
    counts = [(l + BLOCK - 1) // BLOCK for l in lens]
    request = np.repeat(np.arange(len(lens)), counts)
    first = np.concatenate([[0], np.cumsum(counts)])
    place = np.arange(len(request)) - first[request]
    start = np.concatenate([[0], np.cumsum(lens)])[request]
    local = place[:, None] * BLOCK + np.arange(BLOCK)
    there = local < np.asarray(lens)[request][:, None]
    rows = np.where(there, start[:, None] + local, 0)
    give = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return give(rows), give(there), give(request), give(place), give(first)


def _plain_select(state):
    case = state["case"]
    heads, dim = case["heads"], case["dim"]
    q_rows, q_there, q_req, _, _ = _grid(state["q_lens"])
    k_rows, k_there, k_req, k_place, k_first = _grid(state["kv_lens"])

    def mean(x, rows, there):                                         # [heads, blocks, dim], 64 bits
        x = x[rows].double() * there[:, :, None]
        return (x.sum(1) / there.sum(1, keepdim=True)).reshape(len(rows), heads, dim).transpose(0, 1)

    scores = mean(state["q"], q_rows, q_there) @ mean(state["k"], k_rows, k_there).transpose(1, 2)
    limit = torch.tensor(state["kv_lens"], device="cuda")
    tail = torch.tensor(state["tail"], device="cuda")
    kept = (k_place + 1) * BLOCK > (limit - tail)[k_req]              # holds one of the request's last rows
    scores = torch.where(kept & (tail[k_req] > 0), math.inf, scores)
    scores = torch.where(q_req[:, None] == k_req[None, :], scores, -math.inf)
    order = torch.sort(scores, dim=2, descending=True, stable=True).indices
    n_blocks = (limit + BLOCK - 1) // BLOCK
    count = torch.minimum(torch.tensor(state["keep"], device="cuda"), n_blocks)[q_req]
    width = max(state["keep"])
    order = torch.nn.functional.pad(order, (0, max(0, width - order.shape[2])))[:, :, :width] - k_first[q_req][None, :, None]
    taken = torch.arange(width, device="cuda")[None, :] < count[:, None]
    index = torch.where(taken, order, 1 << 40).sort(dim=2).values
    index = torch.where(taken, index, -1).int()
    return index, count.int()[None].expand(heads, -1).contiguous()


def _plain_attend(state):
    case = state["case"]
    heads, dim = case["heads"], case["dim"]
    q_rows, q_there, q_req, _, _ = _grid(state["q_lens"])
    k_rows, k_there, _, _, k_first = _grid(state["kv_lens"])
    deep = min(BLOCK, max(state["q_lens"]))
    q_rows, q_there = q_rows[:, :deep], q_there[:, :deep]

    def blocks(x, rows, there):                                       # [heads, blocks, rows, dim]
        return (x[rows].float() * there[:, :, None]).reshape(*rows.shape, heads, dim).permute(2, 0, 1, 3)

    q, k, v = blocks(state["q"], q_rows, q_there), blocks(state["k"], k_rows, k_there), blocks(state["v"], k_rows, k_there)
    index, count = state["index"].long(), state["count"]
    taken = torch.arange(index.shape[2], device="cuda") < count[:, :, None]
    at = torch.where(taken, index + k_first[q_req][None, :, None], 0)
    head = torch.arange(heads, device="cuda")[:, None, None]
    there = (taken[..., None] & k_there[at]).flatten(2)[:, :, None, :]                    # [heads, query blocks, 1, keys]
    scores = q @ k[head, at].flatten(2, 3).transpose(2, 3) / math.sqrt(dim)
    scores = torch.where(there, scores, -math.inf)
    top = scores.amax(3, keepdim=True)
    p = torch.exp(scores - torch.where(top > -math.inf, top, 0.0))
    total = p.sum(3, keepdim=True)
    out = (p @ v[head, at].flatten(2, 3)) / torch.where(total > 0, total, 1.0)
    out = out.permute(1, 2, 0, 3).flatten(2)                                              # [query blocks, rows, heads * dim]
    return out[q_there].to(TYPES[case["type"]])


# --------------------------------------------------------------------------------------------- one pass
def run(state):
    case = state["case"]
    if case["op"] == "quantize":
        if own:
            from paper_2510_01565_b200 import binding as B
            codes, scales = B.dit_quantize_weight_block128(state["x"]) if case["weight"] else B.dit_quantize_block128(state["x"])
            return {"codes": codes, "scales": scales}
        return _plain_quantize(state)
    if case["op"] == "gemm":
        if own:
            from paper_2510_01565_b200 import binding as B
            return B.dit_gemm_block128(state["a"], state["a_scale"], state["b"], state["b_scale"], bias=state["bias"],
                                       out_dtype=TYPES[case["out"]])
        return _plain_gemm(state)
    if case["op"] == "select":
        if own:
            from paper_2510_01565_b200 import binding as B
            return B.dit_select_blocks(state["q"], state["k"], state["q_lens"], state["kv_lens"], case["heads"], state["keep"],
                                       tail_rows=state["tail"])
        return _plain_select(state)
    if own:
        from paper_2510_01565_b200 import binding as B
        return B.dit_block_attention(state["q"], state["k"], state["v"], state["q_lens"], state["kv_lens"], case["heads"],
                                     state["index"], state["count"])
    return _plain_attend(state)


def work(case):
    if case["op"] == "quantize":
        n = case["rows"] * case["cols"]
        scales = (case["rows"] if not case["weight"] else (case["rows"] + BLOCK - 1) // BLOCK) * ((case["cols"] + BLOCK - 1) // BLOCK)
        return {"bytes": n * (SIZE[case["type"]] + 1) + 4 * scales, "flops": 3 * n}
    if case["op"] == "gemm":
        m, n, k = case["m"], case["n"], case["k"]
        kb, nb = (k + BLOCK - 1) // BLOCK, (n + BLOCK - 1) // BLOCK
        return {"bytes": m * k + n * k + 4 * (kb * m + kb * nb) + (4 * n if case["bias"] else 0) + m * n * SIZE[case["out"]],
                "flops": 2 * m * n * k}
    q_lens, kv_lens = _lens(case["q_lens"]), _lens(case["kv_lens"])
    heads, dim, width = case["heads"], case["dim"], case["heads"] * case["dim"]
    counts = [(q, l, (q + BLOCK - 1) // BLOCK, (l + BLOCK - 1) // BLOCK) for q, l in zip(q_lens, kv_lens)]
    lists = 4 * heads * sum(qb * (case["keep"] + 1) for _, _, qb, _ in counts)
    if case["op"] == "select":
        return {"bytes": 2 * width * (sum(q_lens) + sum(kv_lens)) + lists,
                "flops": width * (sum(q_lens) + sum(kv_lens)) + 2 * width * sum(qb * kb for _, _, qb, kb in counts)}
    keys = [min(l, BLOCK * case["keep"]) for l in kv_lens]
    # of k and v no more than the selected blocks is needed: all of them where many query blocks select
    read = sum(min(l, qb * s) for (_, l, qb, _), s in zip(counts, keys))
    return {"bytes": 2 * width * (2 * sum(q_lens) + 2 * read) + lists, "flops": 4 * width * sum(q * s for q, s in zip(q_lens, keys))}


# --------------------------------------------------------------------------------------------- the definitions, in 64 bits
def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] == "quantize":
        x = state["x"].double()
        if case["weight"]:
            x = x.t()
        rows, cols = x.shape
        row = torch.arange(rows, device="cuda") // (BLOCK if case["weight"] else 1)
        n_col = (cols + BLOCK - 1) // BLOCK
        where = (row[:, None] * n_col + torch.arange(cols, device="cuda")[None, :] // BLOCK)
        top = torch.full((int(row[-1]) + 1, n_col), FLOOR, device="cuda", dtype=torch.float64)
        top.view(-1).scatter_reduce_(0, where.flatten(), x.abs().flatten(), "amax")
        ratio = x * E4M3_MAX / top.view(-1)[where]
        # the nearest value of the format: three bits after the leading one, steps of 2^-9 below 2^-6
        step = torch.exp2(torch.floor(torch.log2(ratio.abs().clamp(min=2.0 ** -6))) - 3)
        codes = torch.round(ratio / step) * step
        scales = top / E4M3_MAX
        return {"codes": codes, "scales": scales if case["weight"] else scales.t()}
    if case["op"] == "gemm":
        out = torch.zeros(case["m"], case["n"], device="cuda", dtype=torch.float64)
        for i in range((case["k"] + BLOCK - 1) // BLOCK):              # block after block, each product scaled as it is added
            cols = slice(i * BLOCK, min(case["k"], (i + 1) * BLOCK))
            part = state["a"][:, cols].to(torch.float64) @ state["b"][:, cols].to(torch.float64).t()
            by_col = state["b_scale"][:, i].double().repeat_interleave(BLOCK)[:case["n"]]
            out += part * state["a_scale"][i].double()[:, None] * by_col[None, :]
        return out if state["bias"] is None else out + state["bias"].double()
    heads, dim = case["heads"], case["dim"]
    q0 = np.concatenate([[0], np.cumsum(state["q_lens"])])
    k0 = np.concatenate([[0], np.cumsum(state["kv_lens"])])
    if case["op"] == "select":
        return None                                                    # whole numbers: there is no error to state
    index, count = state["index"].cpu().numpy(), state["count"].cpu().numpy()
    out = torch.zeros(sum(state["q_lens"]), heads * dim, device="cuda", dtype=torch.float64)
    block = 0
    for r, (ql, kl) in enumerate(zip(state["q_lens"], state["kv_lens"])):
        for first in range(0, ql, BLOCK):
            rows = slice(q0[r] + first, q0[r] + min(ql, first + BLOCK))
            # every head's list as a mask over the request's keys
            seen = np.zeros((heads, (kl + BLOCK - 1) // BLOCK), dtype=bool)
            for h in range(heads):
                seen[h, index[h, block, :count[h, block]]] = True
            seen = torch.from_numpy(np.repeat(seen, BLOCK, axis=1)[:, :kl]).cuda()
            split = lambda t, s: t[s].double().reshape(-1, heads, dim).transpose(0, 1)
            keys = slice(k0[r], k0[r + 1])
            s = split(state["q"], rows) @ split(state["k"], keys).transpose(1, 2) * dim ** -0.5
            p = torch.softmax(s.masked_fill(~seen[:, None, :], -math.inf), dim=2)
            out[rows] = (p @ split(state["v"], keys)).transpose(0, 1).reshape(-1, heads * dim)
            block += 1
    return out

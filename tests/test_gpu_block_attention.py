"""Attention over selected key blocks and the selector, against plain evaluations in 64 bits.

Selected lists are compared for equality (both sides score in 64 bits).  The attention's error is counted from its
arithmetic, with eps the spacing of the inputs' type (fp16 2^-10, bf16 2^-7) and one row's results o = sum p v / sum p:
  * a probability is rounded to the inputs' type (eps / 2) and its exponential comes from scores that fp32 sums of d
    products give with an error of at most (d + 2) * 2^-23 * scale * sum |q k| (natural units), plus 2^-21 for the
    hardware's exp2; both enter numerator and denominator (the denominator without the rounding), so the result is off by at most
    2 * (score error + 2^-21) + eps / 2 of sum p |v| / sum p;
  * probabilities below the type's smallest normal number (fp16: 2^-14 of the largest, times up to 2^8 of head room) lose
    up to 2^-25 each: n keys lose at most n * 2^-25 * max |v|;
  * sums over n keys are fp32: n * 2^-23 of sum p |v| / sum p at most;
  * the output is rounded once: eps / 2 of it, or half the smallest subnormal.
"""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("these tests need a CUDA device; the library has no CPU path")
    from paper_2510_01565_b200 import binding, build
    build.build_library()
    binding.load_library()
    return binding


def blocks_of(n):
    return (n + 127) // 128


def draw(seed, q_lens, kv_lens, heads, dim, kind, sharp=1.0):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda rows: torch.randn(rows, heads * dim, generator=g, device="cuda")
    return tuple(t.to(getattr(torch, kind)) for t in (n(sum(q_lens)) * sharp, n(sum(kv_lens)), n(sum(kv_lens))))


def random_lists(seed, q_lens, kv_lens, heads, width, empty=0.1):
    """Lists of random lengths in random order, some entries repeated, some outside the request, some lists empty."""
    import torch
    rng = np.random.default_rng(seed)
    n_q = sum(blocks_of(l) for l in q_lens)
    index = rng.integers(-3, 2 ** 31 - 1, size=(heads, n_q, width)).astype(np.int32)     # behind the count: anything
    count = np.zeros((heads, n_q), np.int32)
    b = 0
    for ql, kl in zip(q_lens, kv_lens):
        for _ in range(blocks_of(ql)):
            for h in range(heads):
                n = 0 if rng.random() < empty else int(rng.integers(1, width + 1))
                index[h, b, :n] = rng.integers(0, max(1, blocks_of(kl)), size=n)
                if n and rng.random() < 0.3:
                    index[h, b, rng.integers(0, n)] = rng.choice([-1, -2 ** 31, blocks_of(kl), 2 ** 31 - 1])
                count[h, b] = n
            b += 1
    return torch.from_numpy(index).cuda(), torch.from_numpy(count).cuda()


def plain(q, k, v, q_lens, kv_lens, heads, index, count, scale=0.0):
    """(result, allowed error) in 64 bits."""
    import torch
    width = q.shape[1]
    dim = width // heads
    scale = scale or dim ** -0.5
    eps = torch.finfo(q.dtype).eps
    out, room = torch.zeros(q.shape, dtype=torch.float64, device="cuda"), torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    index, count = index.cpu().numpy(), count.cpu().numpy()
    b = q0 = k0 = 0
    for ql, kl in zip(q_lens, kv_lens):
        for first in range(0, ql, 128):
            rows = slice(q0 + first, q0 + min(ql, first + 128))
            for h in range(heads):
                cols = slice(h * dim, (h + 1) * dim)
                chosen = sorted({int(j) for j in index[h, b, :max(0, min(count[h, b], index.shape[2]))] if 0 <= j < blocks_of(kl)})
                keys = torch.tensor([k0 + i for j in chosen for i in range(128 * j, min(kl, 128 * j + 128))], dtype=torch.long, device="cuda")
                if len(keys) == 0:
                    continue
                x, y, z = q[rows, cols].double(), k[keys, cols].double(), v[keys, cols].double()
                s = scale * (x @ y.t())
                s_err = (dim + 2) * 2.0 ** -23 * scale * (x.abs() @ y.abs().t()).amax(1, keepdim=True)
                p = torch.softmax(s, dim=1)
                out[rows, cols] = p @ z
                mag = p @ z.abs()
                n = len(keys)
                room[rows, cols] = mag * (2 * (s_err + 2.0 ** -21) + eps / 2 + n * 2.0 ** -23) + n * 2.0 ** -25 * z.abs().amax()
            b += 1
        q0, k0 = q0 + ql, k0 + kl
    room += eps / 2 * (out.abs() + room) + (2.0 ** -25 if q.dtype == torch.float16 else 0.0)
    return out, room


def check(got, want):
    out, room = want
    off = (got.double() - out).abs()
    assert bool((off <= room).all()), f"off by {float((off / room.clamp(min=1e-30)).max()):.2f} of what is allowed"


BATCHES = [([1], [1]), ([1], [128]), ([1], [1000]), ([3, 1, 0, 4], [129, 5000, 77, 0]), ([2, 2], [300, 4096]), ([5], [40]), ([16, 9], [700, 64]), ([17], [400]), ([128], [128]), ([129], [129]),
           ([130, 1, 257], [130, 1, 257]), ([300, 40, 0, 512], [1000, 0, 50, 700]), ([200, 3], [0, 0]), ([4], [0]), ([640], [2300])]


@pytest.mark.parametrize("q_lens,kv_lens", BATCHES)
@pytest.mark.parametrize("kind,dim,heads", [("float16", 128, 3), ("bfloat16", 128, 2), ("float16", 64, 2), ("bfloat16", 64, 5)])
def test_attention_over_any_lists(B, q_lens, kv_lens, kind, dim, heads):
    import torch
    seed = sum(q_lens) + 7 * sum(kv_lens) + dim + heads
    q, k, v = draw(seed, q_lens, kv_lens, heads, dim, kind, sharp=2.0)
    index, count = random_lists(seed, q_lens, kv_lens, heads, 9)
    out = torch.full_like(q, float("nan"))
    B.dit_block_attention(q, k, v, q_lens, kv_lens, heads, index, count, out=out)
    B.dit_ops_poll_status()
    check(out, plain(q, k, v, q_lens, kv_lens, heads, index, count))


@pytest.mark.parametrize("q_lens", [[2], [200]])
def test_all_blocks_listed_is_dense_attention(B, q_lens):
    import torch
    kv_lens, heads, dim = [3000], 2, 128
    q, k, v = draw(5, q_lens, kv_lens, heads, dim, "float16")
    n_q, n_k = blocks_of(q_lens[0]), blocks_of(3000)
    index = torch.arange(n_k, dtype=torch.int32, device="cuda").flip(0).expand(heads, n_q, n_k).contiguous()
    count = torch.full((heads, n_q), n_k, dtype=torch.int32, device="cuda")
    for scale in (0.0, 0.5):
        out = B.dit_block_attention(q, k, v, q_lens, kv_lens, heads, index, count, scale=scale)
        check(out, plain(q, k, v, q_lens, kv_lens, heads, index, count, scale))
        s = torch.einsum("qhd,khd->hqk", q.double().view(-1, heads, dim), k.double().view(-1, heads, dim)) * (scale or dim ** -0.5)
        dense = torch.einsum("hqk,khd->qhd", torch.softmax(s, 2), v.double().view(-1, heads, dim)).reshape(q.shape)
        assert float((out.double() - dense).abs().max()) <= float(plain(q, k, v, q_lens, kv_lens, heads, index, count, scale)[1].max())


@pytest.mark.parametrize("rows", [1, 13, 140])
def test_more_key_blocks_than_one_window(B, rows):
    """70000 keys (547 blocks: three windows of the tiled kernel), lists that reach into all of them, into the last only, or the first."""
    import torch
    heads, dim, kv = 2, 64, 70000
    q, k, v = draw(17, [rows], [kv], heads, dim, "float16")
    n_q = blocks_of(rows)
    index = torch.full((heads, n_q, 6), -1, dtype=torch.int32, device="cuda")
    index[0, 0] = torch.tensor([546, 3, 511, 512, 3, 600])
    index[1, 0] = torch.tensor([530, 513, 514, 0, 0, 0])
    if n_q > 1:
        index[0, 1] = torch.tensor([512, 2, 545, 0, 0, 0])
        index[1, 1] = torch.tensor([9, 8, 7, 0, 0, 0])
    count = torch.full((heads, n_q), 3, dtype=torch.int32, device="cuda")
    count[0, 0] = 6
    out = B.dit_block_attention(q, k, v, [rows], [kv], heads, index, count)
    B.dit_ops_poll_status()
    check(out, plain(q, k, v, [rows], [kv], heads, index, count))


@pytest.mark.parametrize("q_lens,kv_lens", [([3, 2, 1], [130, 60, 300]), ([130, 60, 300], [130, 60, 300])])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -65504.0])
def test_other_requests_and_unlisted_blocks_may_hold_anything(B, q_lens, kv_lens, bad):
    """Request 1's keys and values are NaN, infinite or extreme, and so is a block of request 2 that nobody lists: requests 0
    and 2 come out as when those are zero, though their last tiles reach into the neighbours' rows."""
    import torch
    heads, dim = 2, 128
    q, k, v = draw(23, q_lens, kv_lens, heads, dim, "float16")
    n_q = sum(blocks_of(l) for l in q_lens)
    index = torch.zeros((heads, n_q, 2), dtype=torch.int32, device="cuda")
    index[:, :, 1] = torch.tensor(sum(([blocks_of(kl) - 1] * blocks_of(ql) for ql, kl in zip(q_lens, kv_lens)), []), dtype=torch.int32, device="cuda")
    count = torch.full((heads, n_q), 2, dtype=torch.int32, device="cuda")
    hidden = [slice(130, 190), slice(190 + 128, 190 + 256)]                       # request 1, block 1 of request 2
    for s in hidden:
        k[s], v[s] = 0.0, 0.0
    clean = B.dit_block_attention(q, k, v, q_lens, kv_lens, heads, index, count)
    for s in hidden:
        k[s], v[s] = bad, bad
    got = B.dit_block_attention(q, k, v, q_lens, kv_lens, heads, index, count)
    own = list(range(q_lens[0])) + list(range(q_lens[0] + q_lens[1], sum(q_lens)))
    assert torch.equal(got[own], clean[own]) and bool(got[own].isfinite().all())


@pytest.mark.parametrize("q_lens", [[3], [140]])
def test_a_nan_in_a_listed_block_is_not_hidden(B, q_lens):
    import torch
    q, k, v = draw(29, q_lens, [500], 1, 64, "bfloat16")
    index = torch.tensor([[[0, 3]] * blocks_of(q_lens[0])], dtype=torch.int32, device="cuda")
    count = torch.full((1, blocks_of(q_lens[0])), 2, dtype=torch.int32, device="cuda")
    v[400, 5] = float("nan")
    out = B.dit_block_attention(q, k, v, q_lens, [500], 1, index, count)
    assert bool(out[:, 5].isnan().all()) and bool(out[:, :5].isfinite().all()) and bool(out[:, 6:].isfinite().all())
    k[10] = float("nan")
    assert bool(B.dit_block_attention(q, k, v, q_lens, [500], 1, index, count).isnan().all())


@pytest.mark.parametrize("q_lens", [[4, 2], [150, 20]])
def test_scores_far_apart(B, q_lens):
    """Scores of several hundred (one key of a row takes everything), growing along the list, so that the running reference moves."""
    import torch
    heads, dim, kv_lens = 2, 64, [1000, 300]
    q, k, v = draw(31, q_lens, kv_lens, heads, dim, "float16", sharp=8.0)
    k[:1000] *= torch.linspace(0.1, 6.0, 1000, device="cuda")[:, None].half()
    n_q = sum(blocks_of(l) for l in q_lens)
    index = torch.arange(8, dtype=torch.int32, device="cuda").expand(heads, n_q, 8).contiguous()
    count = torch.full((heads, n_q), 8, dtype=torch.int32, device="cuda")
    out = B.dit_block_attention(q, k, v, q_lens, kv_lens, heads, index, count)
    check(out, plain(q, k, v, q_lens, kv_lens, heads, index, count))


@pytest.mark.parametrize("q_lens", [[4, 3], [140, 3]])
def test_strided_inputs_and_an_output_inside_a_wider_buffer(B, q_lens):
    import torch
    heads, dim, kv_lens = 3, 64, [200, 333]
    width = heads * dim
    q, k, v = draw(37, q_lens, kv_lens, heads, dim, "bfloat16")
    index, count = random_lists(37, q_lens, kv_lens, heads, 3)
    wide_q = torch.full((sum(q_lens), width + 16), float("nan"), dtype=q.dtype, device="cuda")
    wide_q[:, 8:8 + width] = q
    kv = torch.full((sum(kv_lens), 2 * width + 8), float("nan"), dtype=q.dtype, device="cuda")
    kv[:, :width], kv[:, width:2 * width] = v, k
    buf = torch.full((sum(q_lens) + 2, width + 24), 7.0, dtype=q.dtype, device="cuda")
    out = buf[1:-1, 16:16 + width]
    B.dit_block_attention(wide_q[:, 8:8 + width], kv[:, width:2 * width], kv[:, :width], q_lens, kv_lens, heads, index, count, out=out)
    check(out, plain(q, k, v, q_lens, kv_lens, heads, index, count))
    rest = buf.clone()
    rest[1:-1, 16:16 + width] = 7.0
    assert bool((rest == 7.0).all())


def test_more_heads_and_requests_than_ctas_and_packed_equals_alone(B):
    import torch
    heads, dim = 5, 64
    q_lens = [1 + (37 * i) % 300 for i in range(64)]
    kv_lens = [1 + (91 * i) % 700 for i in range(64)]
    q, k, v = draw(41, q_lens, kv_lens, heads, dim, "float16")
    keep = [1 + i % 4 for i in range(64)]
    index, count = B.dit_select_blocks(q, k, q_lens, kv_lens, heads, keep)
    out = B.dit_block_attention(q, k, v, q_lens, kv_lens, heads, index, count)
    check(out, plain(q, k, v, q_lens, kv_lens, heads, index, count))
    q0 = k0 = b0 = 0
    for r in range(64):
        qs, ks, bs = slice(q0, q0 + q_lens[r]), slice(k0, k0 + kv_lens[r]), slice(b0, b0 + blocks_of(q_lens[r]))
        i1, c1 = B.dit_select_blocks(q[qs], k[ks], [q_lens[r]], [kv_lens[r]], heads, [keep[r]])
        assert torch.equal(i1, index[:, bs, :keep[r]]) and torch.equal(c1, count[:, bs])
        if q_lens[r] > 16:     # up to sixteen rows alone go through the other kernel
            assert torch.equal(B.dit_block_attention(q[qs], k[ks], v[ks], [q_lens[r]], [kv_lens[r]], heads, i1, c1), out[qs])
        q0, k0, b0 = q0 + q_lens[r], k0 + kv_lens[r], b0 + blocks_of(q_lens[r])


# ------------------------------------------------------------------------------------------------ the selector
def plain_select(q, k, q_lens, kv_lens, heads, keep, tail):
    dim = q.shape[1] // heads
    q, k = q.double().cpu().numpy(), k.double().cpu().numpy()
    widest = max(keep)
    index, count = [], []
    q0 = k0 = 0
    for r, (ql, kl) in enumerate(zip(q_lens, kv_lens)):
        km = [k[k0 + 128 * j:k0 + min(kl, 128 * j + 128)].mean(0) for j in range(blocks_of(kl))]
        for i in range(blocks_of(ql)):
            qm = q[q0 + 128 * i:q0 + min(ql, 128 * i + 128)].mean(0)
            lists, counts = [], []
            for h in range(heads):
                c = slice(h * dim, (h + 1) * dim)
                s = [math.inf if tail[r] > 0 and (j + 1) * 128 > kl - tail[r] else float(qm[c] @ km[j][c]) for j in range(len(km))]
                best = sorted(sorted(range(len(km)), key=lambda j: (-s[j], j))[:keep[r]])
                lists.append(best + [-1] * (widest - len(best)))
                counts.append(len(best))
            index.append(lists)
            count.append(counts)
        q0, k0 = q0 + ql, k0 + kl
    return np.array(index, np.int32).transpose(1, 0, 2), np.array(count, np.int32).T


@pytest.mark.parametrize("q_lens,kv_lens,keep,tail", [([1], [1], [1], [0]), ([5], [1000], [3], [0]), ([300, 0, 129], [1500, 400, 0], [4, 2, 5], [77, 0, 9]),
                                                      ([513], [5000], [40], [512]), ([200], [1290], [2], [700]), ([130, 20], [130, 2600], [1, 21], [500, 1])])
@pytest.mark.parametrize("kind,dim,heads", [("float16", 128, 3), ("bfloat16", 64, 5), ("float16", 64, 1)])
def test_selection_equals_the_plain_one(B, q_lens, kv_lens, keep, tail, kind, dim, heads):
    q, k, _ = draw(sum(kv_lens) + dim, q_lens, kv_lens, heads, dim, kind)
    index, count = B.dit_select_blocks(q, k, q_lens, kv_lens, heads, keep, tail_rows=tail)
    want_index, want_count = plain_select(q, k, q_lens, kv_lens, heads, keep, tail)
    assert np.array_equal(index.cpu().numpy(), want_index) and np.array_equal(count.cpu().numpy(), want_count)


def test_selection_among_equal_scores_takes_the_lowest_blocks(B):
    import torch
    heads, dim = 2, 64
    q = torch.ones(128, heads * dim, dtype=torch.float16, device="cuda")
    k = torch.zeros(128 * 40, heads * dim, dtype=torch.float16, device="cuda")
    k[128 * 30:128 * 35] = 1.0                                         # five equal scores above thirty-five equal ones
    k[128 * 7:128 * 8, :] = -0.0                                       # a negative zero is a zero
    for keep in (1, 3, 5, 6, 12, 40):
        index, count = B.dit_select_blocks(q, k, [128], [128 * 40], heads, [keep])
        best = list(range(30, 30 + min(5, keep))) + [j for j in range(40) if not 30 <= j < 35][:max(0, keep - 5)]
        assert index[0, 0].tolist() == sorted(best) and index[1, 0].tolist() == sorted(best) and count.flatten().tolist() == [keep, keep]
    k[128 * 3] = float("nan")                                          # counts as less than any number
    index, _ = B.dit_select_blocks(q, k, [128], [128 * 40], heads, [39])
    assert index[0, 0].tolist() == [j for j in range(40) if j != 3]


def test_selection_with_many_key_blocks(B):
    """3000 key blocks: lists longer than a warp's stride, one query block per CTA group, scores from a few rows' means."""
    import torch
    heads, dim, kv = 1, 64, 128 * 3000 - 17
    q, k, _ = draw(43, [400], [kv], heads, dim, "float16")
    index, count = B.dit_select_blocks(q, k, [400], [kv], heads, [777], tail_rows=[300])
    qm = torch.stack([q[128 * i:128 * i + 128].double().mean(0) for i in range(4)])
    km = torch.nn.functional.pad(k.double(), (0, 0, 0, 17)).view(3000, 128, dim).sum(1)
    km[:-1] /= 128
    km[-1] /= 128 - 17
    s = qm @ km.t()
    s[:, 3000 - 3:] = math.inf                                         # blocks of the last 300 rows
    want = s.topk(777, dim=1).indices.sort(dim=1).values.int()
    assert torch.equal(index[0], want) and count.tolist() == [[777] * 4]


def test_select_and_attend_on_another_stream_and_in_a_graph(B):
    import torch
    heads, dim, q_lens = 3, 128, [400, 77]
    q, k, v = draw(47, q_lens, q_lens, heads, dim, "float16")

    def both():
        index, count = B.dit_select_blocks(q, k, q_lens, q_lens, heads, [2, 1])
        return index, B.dit_block_attention(q, k, v, q_lens, q_lens, heads, index, count)
    first = both()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = both()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, second))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        third = both()
    q.copy_(-q)
    graph.replay()
    want = both()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(third, want)) and not torch.equal(first[1], third[1])


# ------------------------------------------------------------------------------------------------ scores and values at the format's edges
def whole_numbers(seed, q_lens, kv_lens, heads, dim, kind, unit, offset):
    """q and k of small whole numbers times `unit`, every other row of q louder by powers of two, and a channel that shifts all of a row's
    scores alike: products and their sums are whole multiples of unit^2 below 2^24, which fp32 holds without rounding in any order."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda rows: torch.randint(-2, 3, (rows, heads * dim), generator=g, device="cuda").float()
    q, k, v = n(sum(q_lens)), n(sum(kv_lens)), torch.randn(sum(kv_lens), heads * dim, generator=g, device="cuda")
    q[:, ::dim], k[:, ::dim] = 30.0 * (offset != 0), float(offset)
    q *= torch.exp2((torch.arange(len(q), device="cuda") % 4).float() * (torch.arange(len(q), device="cuda") % 2))[:, None]
    t = getattr(torch, kind)
    return (q * unit).to(t), (k * unit).to(t), v.to(t)


def exact_scores(q, k, v, q_lens, kv_lens, heads, index, count, scale):
    """(result, allowed error) in 64 bits where the scores are exact.  What is left of the error, in natural units of the exponent: the factor
    scale * log2 e (off by 2^-22 of itself, with exponents of at most 40 where a probability counts: 40 * 2^-22), the hardware's exp2 (2^-21), and
    a reference rounded after scaling while it is below 2^10 (2^-14, for two references of one row 2^-13); below 2^-12 together.
    Then as for `plain`: probabilities and result rounded to the inputs' type, sums in fp32, the smallest probabilities."""
    import torch
    dim, eps = q.shape[1] // heads, torch.finfo(q.dtype).eps
    scale = float(np.float32(scale or np.float32(1.0) / np.sqrt(np.float32(dim))))
    out, room = torch.zeros(q.shape, dtype=torch.float64, device="cuda"), torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    b = q0 = k0 = 0
    for ql, kl in zip(q_lens, kv_lens):
        for first in range(0, ql, 128):
            rows = slice(q0 + first, q0 + min(ql, first + 128))
            for h in range(heads):
                cols = slice(h * dim, (h + 1) * dim)
                chosen = sorted(set(index[h, b, :int(count[h, b])].tolist()))
                keys = torch.tensor([k0 + i for j in chosen for i in range(128 * j, min(kl, 128 * j + 128))], dtype=torch.long, device="cuda")
                s = scale * (q[rows, cols].double() @ k[keys, cols].double().t())
                p, z = torch.softmax(s, dim=1), v[keys, cols].double()
                out[rows, cols], mag, n = p @ z, p @ z.abs(), len(keys)
                room[rows, cols] = mag * (2 * 2.0 ** -12 + eps / 2 + n * 2.0 ** -23) + n * 2.0 ** -25 * z.abs().amax()
            b += 1
        q0, k0 = q0 + ql, k0 + kl
    room += eps / 2 * (out.abs() + room) + (2.0 ** -25 if q.dtype == torch.float16 else 0.0)
    return out, room


@pytest.mark.parametrize("q_lens", [[3, 16], [140, 16]])
@pytest.mark.parametrize("kind,dim,unit,scale", [("float16", 64, 1.0, s) for s in (0.0, 2.0 ** -4, 1e4, 1e6, 1e8, 1e12, 2e38)]
                         + [("bfloat16", 128, 1.0, s) for s in (1e8, 2e38)]
                         + [("float16", 128, 2048.0, 0.0), ("bfloat16", 64, 2.0 ** 20, 0.0), ("bfloat16", 128, 2.0 ** 56, 0.0), ("bfloat16", 64, 2.0 ** 54, 1.0)])
@pytest.mark.parametrize("offset", [0, 30, -30])
def test_large_scaled_scores(B, q_lens, kind, dim, unit, scale, offset):
    """Scaled scores of any size fp32 holds, and factors up to the largest that is accepted: the largest keys of a row share its result, whatever
    the sign of their scores.  (An exponent formed as s * c - round(m * c) is off by the rounding of m * c, which is 16 at 2^28 and
    infinite soon after 2^128: the row then came out as zeros.)"""
    import torch
    heads, kv_lens = 2, [700, 300]
    if kind == "float16" and unit > 1 and offset:
        unit /= 32.0                                                    # 30 * 8 * unit has to stay below 65504
    q, k, v = whole_numbers(71 + dim, q_lens, kv_lens, heads, dim, kind, unit, offset)
    n_q = sum(blocks_of(l) for l in q_lens)
    index = torch.tensor([5, 0, 2], dtype=torch.int32, device="cuda").expand(heads, n_q, 3).contiguous()
    index[:, -1] = torch.tensor([2, 0, 1], dtype=torch.int32)
    count = torch.full((heads, n_q), 3, dtype=torch.int32, device="cuda")
    out = B.dit_block_attention(q, k, v, q_lens, kv_lens, heads, index, count, scale=scale)
    B.dit_ops_poll_status()
    check(out, exact_scores(q, k, v, q_lens, kv_lens, heads, index, count, scale))


@pytest.mark.parametrize("q_lens", [[3, 16], [140, 16]])
@pytest.mark.parametrize("kind", ["float16", "bfloat16"])
def test_an_infinity_in_a_listed_block_is_not_hidden(B, q_lens, kind):
    """As in the definition, an infinite value makes its channel infinite, and two of opposite signs a NaN; a channel at the type's largest
    value stays there although the rounded probabilities may add up to a little more than one."""
    import torch
    heads, dim, kv_lens = 1, 64, [300, 200]
    q, k, v = draw(73, q_lens, kv_lens, heads, dim, kind, sharp=0.25)   # every probability is far above what rounds to zero
    n_q = sum(blocks_of(l) for l in q_lens)
    index = torch.tensor([[[0, 2]] * (n_q - 1) + [[0, 1]]], dtype=torch.int32, device="cuda")
    count = torch.full((1, n_q), 2, dtype=torch.int32, device="cuda")
    v[10], v[300 + 150] = 0.0, 0.0
    clean = B.dit_block_attention(q, k, v, q_lens, kv_lens, heads, index, count)
    inf = float("inf")
    top = 65504.0 if kind == "float16" else 2.0 ** 98
    for r in (10, 300 + 150):
        v[r, 3], v[r, 4], v[r, 5] = inf, -inf, inf
    for r in (11, 300 + 20):
        v[r, 5] = -inf
    v[:, 6], v[:, 7], v[130, :] = top, -top, inf                        # (row 130 belongs to a block that nobody lists)
    out = B.dit_block_attention(q, k, v, q_lens, kv_lens, heads, index, count)
    B.dit_ops_poll_status()
    assert bool((out[:, 3] == inf).all()) and bool((out[:, 4] == -inf).all()) and bool(out[:, 5].isnan().all())
    # top times a weighted mean of ones: off by the probabilities' rounding, the sums' and the result's
    for c, want in ((6, top), (7, -top)):
        assert bool((out[:, c].double() / want - 1.0).abs().max() <= torch.finfo(out.dtype).eps + 2.0 ** -11)
        assert bool(out[:, c].isfinite().all())
    rest = [c for c in range(64) if not 3 <= c <= 7]
    assert torch.equal(out[:, rest], clean[:, rest])

"""Attention over packed requests with grouped heads against a plain evaluation in 64 bits.

The error is counted from the arithmetic, with eps the spacing of the inputs' type (fp16 2^-10, bf16 2^-7) and a row's result
o = sum p v / sum p:
  * a probability is rounded to the inputs' type (eps / 2) and its exponential comes from scores that fp32 sums of d
    products give with an error of at most (d + 2) * 2^-23 * scale * sum |q k| (natural units), plus 2^-21 for the
    hardware's exp2; both enter numerator and denominator (the denominator without the rounding), so the result is off by at most
    2 * (score error + 2^-21) + eps / 2 of sum p |v| / sum p;
  * probabilities below the type's smallest normal number (fp16: 2^-14 of the largest, times up to 2^8 of head room) lose
    up to 2^-25 each: n keys lose at most n * 2^-25 * max |v|;
  * sums over n keys are fp32: n * 2^-23 of sum p |v| / sum p at most;
  * the output is rounded once: eps / 2 of it, or half the smallest subnormal.
"""
import numpy as np
import pytest

from oracle import prompt_oracle as P

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


def draw(seed, q_lens, kv_lens, heads, kv_heads, dim, kind, sharp=1.0):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda rows, h: torch.randn(rows, h * dim, generator=g, device="cuda")
    return tuple(t.to(getattr(torch, kind)) for t in (n(sum(q_lens), heads) * sharp, n(sum(kv_lens), kv_heads), n(sum(kv_lens), kv_heads)))


def plain(q, k, v, q_lens, kv_lens, heads, kv_heads, causal=True, scale=0.0):
    """(result, allowed error) in 64 bits."""
    import torch
    dim = q.shape[1] // heads
    scale = scale or dim ** -0.5
    eps = torch.finfo(q.dtype).eps
    out, room = torch.zeros(q.shape, dtype=torch.float64, device="cuda"), torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    q0 = k0 = 0
    for ql, kl in zip(q_lens, kv_lens):
        last = kl - ql + torch.arange(ql, device="cuda") if causal else torch.full((ql,), kl - 1, device="cuda")
        hidden = torch.arange(kl, device="cuda")[None, :] > last[:, None]
        for h in range(heads if ql and kl else 0):
            cols = slice(h * dim, (h + 1) * dim)
            g = h // (heads // kv_heads)
            kc = slice(g * dim, (g + 1) * dim)
            x, y, z = q[q0:q0 + ql, cols].double(), k[k0:k0 + kl, kc].double(), v[k0:k0 + kl, kc].double()
            s = (scale * (x @ y.t())).masked_fill(hidden, float("-inf"))
            s_err = (dim + 2) * 2.0 ** -23 * scale * (x.abs() @ y.abs().t()).masked_fill(hidden, 0.0).amax(1, keepdim=True)
            p = torch.nan_to_num(torch.softmax(s, dim=1), nan=0.0)          # (a row without keys)
            out[q0:q0 + ql, cols] = p @ z
            n = (~hidden).sum(1, keepdim=True)
            room[q0:q0 + ql, cols] = (p @ z.abs()) * (2 * (s_err + 2.0 ** -21) + eps / 2 + n * 2.0 ** -23) + n * 2.0 ** -25 * z.abs().amax()
        q0, k0 = q0 + ql, k0 + kl
    room += eps / 2 * (out.abs() + room) + (2.0 ** -25 if q.dtype == torch.float16 else 0.0)
    return out, room


def check(got, want):
    out, room = want
    off = (got.double() - out).abs()
    assert bool((off <= room).all()), f"off by {float((off / room.clamp(min=1e-30)).max()):.2f} of what is allowed"


BATCHES = [([24], [3000]), ([100, 31, 5], [700, 4000, 4000]), ([1], [1]), ([1], [128]), ([1], [1000]), ([1, 1, 1], [33000, 1, 700]), ([3, 1, 0, 4], [129, 5000, 77, 0]), ([2, 2], [300, 4096]), ([5], [40]),
           ([16, 9], [700, 64]), ([17], [400]), ([64, 33], [64, 4000]), ([65], [65]), ([77, 256, 5, 333], [77, 256, 5, 333]), ([128], [128]), ([129], [129]),
           ([130, 1, 257], [130, 1, 257]), ([300, 40, 0, 512], [1000, 0, 50, 700]), ([200, 3], [0, 0]), ([4], [0]), ([640], [2300]), ([300, 90], [100, 3]),
           ([500], [501]), ([1100], [1100]), ([3000], [3000]), ([2500, 40], [2500, 9000]), ([700], [6000])]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("kind,dim,heads,kv_heads", [("float16", 128, 3, 3), ("bfloat16", 128, 8, 2), ("float16", 64, 6, 2), ("bfloat16", 64, 5, 1), ("float16", 128, 20, 1)])
@pytest.mark.parametrize("q_lens,kv_lens", BATCHES)
def test_attention(B, q_lens, kv_lens, kind, dim, heads, kv_heads, causal):
    q, k, v = draw(sum(kv_lens) + heads, q_lens, kv_lens, heads, kv_heads, dim, kind, 2.0)
    got = B.dit_prompt_attention(q, k, v, q_lens, kv_lens, heads, kv_heads, causal=causal)
    check(got, plain(q, k, v, q_lens, kv_lens, heads, kv_heads, causal))
    B.dit_ops_poll_status()


def test_the_oracle_says_the_same(B):
    q, k, v = draw(3, [30, 70], [50, 70], 4, 2, 64, "float16")
    want = P.attention(q.cpu().numpy(), k.cpu().numpy(), v.cpu().numpy(), [30, 70], [50, 70], 4, 2)
    out, _ = plain(q, k, v, [30, 70], [50, 70], 4, 2)
    assert np.allclose(out.cpu().numpy(), want, atol=1e-12)


def test_many_requests_and_more_items_than_ctas(B):
    import torch
    q_lens = [1 + (37 * i) % 400 for i in range(64)]
    kv_lens = [l + (i * 53) % 200 if i % 3 else l for i, l in enumerate(q_lens)]
    q, k, v = draw(5, q_lens, kv_lens, 8, 4, 64, "bfloat16")
    got = B.dit_prompt_attention(q, k, v, q_lens, kv_lens, 8, 4)
    check(got, plain(q, k, v, q_lens, kv_lens, 8, 4))
    assert torch.equal(got, B.dit_prompt_attention(q, k, v, q_lens, kv_lens, 8, 4))


def test_single_rows_of_many_requests(B):
    q_lens, kv_lens = [1] * 64, [1 + (911 * i) % 5000 for i in range(64)]
    q, k, v = draw(6, q_lens, kv_lens, 16, 2, 128, "float16")
    check(B.dit_prompt_attention(q, k, v, q_lens, kv_lens, 16, 2), plain(q, k, v, q_lens, kv_lens, 16, 2))


CONTEXTS = [([3000], [3000], 2, 1), ([900], [4000], 2, 2), ([200], [200], 4, 2), ([333], [400], 3, 3), ([1], [300], 4, 2), ([7], [300], 4, 2), ([40], [2000], 4, 4), ([150], [900], 5, 1)]


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("q_len,kv_len,heads,kv_heads", [(a[0], b[0], c, d) for a, b, c, d in CONTEXTS])
@pytest.mark.parametrize("kind", ["float16", "bfloat16"])
def test_what_a_row_does_not_see_may_hold_anything(B, q_len, kv_len, heads, kv_heads, bad, kind):
    """Other requests' rows, and a later key and value of the row's own request: rows in front of it keep their bits, rows that see it do not hide it."""
    import torch
    dim = 128
    q_lens, kv_lens = [90, q_len, 70], [90, kv_len, 70]
    q, k, v = draw(kv_len, q_lens, kv_lens, heads, kv_heads, dim, kind)
    clean = B.dit_prompt_attention(q, k, v, q_lens, kv_lens, heads, kv_heads)
    mine = slice(90, 90 + q_len)
    kx, vx = k.clone(), v.clone()
    for t in (kx, vx):
        t[:90] = bad
        t[90 + kv_len:] = bad
    assert torch.equal(B.dit_prompt_attention(q, kx, vx, q_lens, kv_lens, heads, kv_heads)[mine], clean[mine])
    for key in sorted({kv_len - 1, kv_len - q_len, kv_len - q_len // 2 - 1, max(0, kv_len - q_len - 1)}):
        vx = v.clone()
        vx[90 + key, 5] = bad                  # channel 5 of key head 0
        got = B.dit_prompt_attention(q, k, vx, q_lens, kv_lens, heads, kv_heads)
        sees = torch.arange(q_len, device="cuda") + kv_len - q_len >= key
        hit = torch.zeros(sum(q_lens), heads * dim, dtype=torch.bool, device="cuda")
        for h in range(heads // kv_heads):
            hit[mine, h * dim + 5] = sees
        assert not got[hit].isfinite().any() and torch.equal(got[~hit], clean[~hit])
        if bad != bad:
            assert got[hit].isnan().all()
        kx = k.clone()
        kx[90 + key, :dim] = float("nan")
        got = B.dit_prompt_attention(q, kx, v, q_lens, kv_lens, heads, kv_heads)
        gone = torch.zeros_like(hit)
        gone[mine, :heads // kv_heads * dim] = sees[:, None]
        assert got[gone].isnan().all() and torch.equal(got[~gone], clean[~gone])


@pytest.mark.parametrize("q_lens,kv_lens", [([1, 8], [3000, 500]), ([300], [300]), ([200], [2000])])
def test_scores_far_apart_and_large(B, q_lens, kv_lens):
    """Rows whose maximum grows by hundreds from block to block, and scaled scores beyond 2^20."""
    for sharp, scale in ((60.0, 0.0), (1.0, 3.0e4)):
        q, k, v = draw(11, q_lens, kv_lens, 4, 2, 64, "bfloat16", sharp)
        got = B.dit_prompt_attention(q, k, v, q_lens, kv_lens, 4, 2, scale=scale)
        out, room = plain(q, k, v, q_lens, kv_lens, 4, 2, scale=scale)
        close = room < 0.05 * v.double().abs().amax()                  # (rows between two keys whose scores fp32 cannot tell apart say nothing)
        assert bool(((got.double() - out).abs() <= room)[close].all()) and bool(got.isfinite().all())


def test_a_row_of_minus_infinities(B):
    import torch
    for q_len in (1, 200):
        q, k, v = draw(12, [q_len], [300], 2, 1, 64, "float16")
        k[:, 0] = float("inf")
        q[:, 0] = -1.0
        q[:, 64] = -1.0
        got = B.dit_prompt_attention(q, k, v, [q_len], [300], 2, 1)
        assert not got.any()


def test_strides_and_an_output_inside_a_wider_buffer(B):
    import torch
    for q_lens in ([300, 130], [1, 7], [1, 300]):
        heads, kv_heads, dim = 4, 2, 64
        rows, width = sum(q_lens), (heads + 2 * kv_heads) * dim
        big = torch.randn(rows + 2, width + 24, generator=torch.Generator().manual_seed(1)).half().cuda()
        qkv = big[1:-1, 8:8 + width]
        q, k, v = qkv[:, :heads * dim], qkv[:, heads * dim:(heads + kv_heads) * dim], qkv[:, (heads + kv_heads) * dim:]
        want = plain(q, k, v, q_lens, q_lens, heads, kv_heads)
        for left in (8, 16):
            buf = torch.full((rows + 2, heads * dim + 40), 3.0, dtype=torch.float16, device="cuda")
            out = buf[1:-1, left:left + heads * dim]
            B.dit_prompt_attention(q, k, v, q_lens, q_lens, heads, kv_heads, out=out)
            check(out, want)
            assert (buf[0] == 3).all() and (buf[-1] == 3).all() and (buf[:, :left] == 3).all() and (buf[:, left + heads * dim:] == 3).all()


def test_a_workspace_of_the_callers_and_rows_behind_the_batch(B):
    import ctypes as C
    import torch
    q, k, v = draw(9, [1, 2], [9000, 3000], 8, 2, 128, "float16")
    lens = lambda *x: (C.c_int32 * len(x))(*x)
    out = torch.full((5, 1024), 4.0, dtype=torch.float16, device="cuda")
    a = B.DitPromptAttentionArgs(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), 1024, 256, 256, 1024, 0, 8, 2, 128, 1, 0.0, 2, lens(1, 2), lens(9000, 3000))
    lib = B.load_library()
    need = lib.dit_prompt_attention_workspace(C.byref(a))
    assert need > 0
    work = torch.full((need + 64,), 0xFF, dtype=torch.uint8, device="cuda")
    a.workspace, a.workspace_bytes = work.data_ptr(), need - 1
    assert lib.dit_prompt_attention(C.byref(a), torch.cuda.current_stream().cuda_stream) == 3
    a.workspace_bytes = need
    assert lib.dit_prompt_attention(C.byref(a), torch.cuda.current_stream().cuda_stream) == 0
    assert (work[need:] == 0xFF).all() and (out[3:] == 4).all()
    assert torch.equal(out[:3], B.dit_prompt_attention(q, k, v, [1, 2], [9000, 3000], 8, 2, workspace=torch.empty(need, dtype=torch.uint8, device="cuda")))


def test_offsets_beyond_32_bits(B):
    """600 000 keys of 32 key heads of 128: 2.5e9 elements each of k and v; the far end of the keys decides."""
    import torch
    heads, dim, kv = 32, 128, 600_000
    k, v = (torch.zeros(kv, heads * dim, dtype=torch.float16, device="cuda") for _ in range(2))
    g = torch.Generator(device="cuda").manual_seed(1)
    v[-300:] = torch.randn(300, heads * dim, generator=g, device="cuda").half()
    k[-300:] = 1.0
    for q_rows in (1, 130):
        q = torch.full((q_rows, heads * dim), 8.0, dtype=torch.float16, device="cuda")      # scores 8 sqrt(128) = 90 against 0
        out = B.dit_prompt_attention(q, k, v, [q_rows], [kv], heads)
        seen = torch.arange(q_rows, device="cuda") + 301 - q_rows
        want = v[-300:].double().cumsum(0)[seen - 1] / seen[:, None]
        # probabilities of 1 / n in parts: their sum and the values' sums in fp32, the rounding to fp16
        assert float((out.double() - want).abs().max()) <= 300 * 2.0 ** -23 * 6 + 2.0 ** -11 * float(want.abs().max()) + 2.0 ** -25
    B.dit_ops_poll_status()


def test_another_stream_a_graph_and_two_calls_at_once(B):
    import torch
    q_lens, kv_lens = [1, 300, 2, 40], [8000, 300, 900, 2000]
    q, k, v = draw(15, q_lens, kv_lens, 8, 2, 64, "float16")
    q2, k2, v2 = draw(16, q_lens, kv_lens, 8, 2, 64, "float16")
    call = lambda a, b, c: B.dit_prompt_attention(a, b, c, q_lens, kv_lens, 8, 2)
    want, want2 = call(q, k, v), call(q2, k2, v2)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = call(q, k, v)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = []
    for i in range(20):
        with torch.cuda.stream(streams[i % 2]):
            got.append(call(q, k, v) if i % 2 else call(q2, k2, v2))
    torch.cuda.synchronize()
    assert all(torch.equal(x, want if i % 2 else want2) for i, x in enumerate(got))
    for t, u in ((q, q2), (k, k2), (v, v2)):
        t.copy_(u)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(captured, want2)
    B.dit_ops_poll_status()

"""Attention over packed requests where scaled scores are far beyond the exponential's range.

Scores are whole numbers that fp32 holds exactly, all different, and the scale is a large power of two: the largest score that a row sees has the
probability 1, every other one 0 (a difference of 2^8 or more in the exponent).  A row's result is then the value of that key, bit for bit, and
every element is compared.  The largest score moves on from block to block (rising), stays at the first (falling) or jumps (shuffled),
and lies far above or far below zero, so that references beyond the range are taken off before the scaling and replaced on the way.
"""
import ctypes as C

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


def ranks(order, n, seed):
    """Distinct numbers 1 .. 32767 of n keys."""
    import torch
    if order == "shuffled":
        return torch.randperm(32767, generator=torch.Generator().manual_seed(seed))[:n] + 1
    up = 1 + torch.arange(n) * (32766 // n)
    return up if order == "rising" else up.flip(0)


def workspace_bytes(B, q_lens, kv_lens, heads, kv_heads, dim):
    a = B.DitPromptAttentionArgs()
    n = len(q_lens)
    ql, kl = (C.c_int32 * n)(*q_lens), (C.c_int32 * n)(*kv_lens)
    a.type, a.n_heads, a.n_kv_heads, a.head_dim, a.causal, a.n_requests, a.q_lens, a.kv_lens = 1, heads, kv_heads, dim, 1, n, ql, kl
    return B.load_library().dit_prompt_attention_workspace(C.byref(a))


# a few rows, in one part and in several; tiles of whole pairs; pairs cut into parts (128 rows against a long context, a long prompt)
CASES = [([1, 8], [3000, 500], 4, 2, 64, True), ([1], [200], 4, 2, 128, False), ([1], [20000], 8, 1, 128, True), ([600, 700], [600, 900], 16, 8, 64, False),
         ([1500], [1500], 32, 8, 128, False), ([700], [2000], 16, 8, 128, True), ([128], [30000], 32, 8, 128, True), ([5000], [5000], 2, 1, 64, True)]


@pytest.mark.parametrize("sign,base", [(1.0, 0), (-1.0, 0), (1.0, -32768)])
@pytest.mark.parametrize("order", ["rising", "falling", "shuffled"])
@pytest.mark.parametrize("scale", [2.0 ** 8, 2.0 ** 20, 2.0 ** 100])
@pytest.mark.parametrize("q_lens,kv_lens,heads,kv_heads,dim,parts", CASES)
def test_the_largest_score_decides(B, q_lens, kv_lens, heads, kv_heads, dim, parts, scale, order, sign, base):
    """Scores sign * (rank + base): positive, negative, or negative by the base alone."""
    import torch
    assert (workspace_bytes(B, q_lens, kv_lens, heads, kv_heads, dim) > 0) == parts
    rank = torch.cat([ranks(order, n, n) for n in kv_lens]).cuda()
    k = torch.zeros(sum(kv_lens), kv_heads, dim, dtype=torch.bfloat16, device="cuda")
    k[:, :, 3], k[:, :, dim - 9], k[:, :, 17] = ((rank >> s & 31).to(torch.bfloat16)[:, None] for s in (10, 5, 0))      # rank in digits of 32
    k[:, :, 30] = 1.0
    q = torch.zeros(sum(q_lens), heads, dim, dtype=torch.bfloat16, device="cuda")
    q[:, :, 3], q[:, :, dim - 9], q[:, :, 17], q[:, :, 30] = sign * 1024, sign * 32, sign, sign * base
    v = torch.randn(sum(kv_lens), kv_heads * dim, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").bfloat16()
    got = B.dit_prompt_attention(q.flatten(1), k.flatten(1), v, q_lens, kv_lens, heads, kv_heads, scale=scale)
    B.dit_ops_poll_status()
    score = sign * rank.double()
    q0 = k0 = 0
    for ql, kl in zip(q_lens, kv_lens):
        best = torch.cummax(score[k0:k0 + kl], 0).indices[kl - ql:]                     # of the keys up to each row's own
        want = v[k0 + best].reshape(ql, kv_heads, 1, dim).expand(-1, -1, heads // kv_heads, -1).reshape(ql, heads * dim)
        assert torch.equal(got[q0:q0 + ql], want)
        q0, k0 = q0 + ql, k0 + kl


def test_a_workspace_one_byte_too_small_is_refused(B):
    import torch
    need = workspace_bytes(B, [1], [9000], 8, 1, 64)
    assert need > 0
    q, k = torch.zeros(1, 512, dtype=torch.bfloat16, device="cuda"), torch.zeros(9000, 64, dtype=torch.bfloat16, device="cuda")
    room = torch.empty(need, dtype=torch.uint8, device="cuda")
    with pytest.raises(B.DitError) as e:
        B.dit_prompt_attention(q, k, k, [1], [9000], 8, 1, workspace=room[:-1])
    assert e.value.status == 3                                                          # DIT_ERR_CAPACITY
    assert not B.dit_prompt_attention(q, k, k, [1], [9000], 8, 1, workspace=room).any()

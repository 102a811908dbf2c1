"""How attention over packed prompts lays a batch out on the host: what it costs a call, and that a call from Python does it once.  No GPU: only sizes
are read."""
import ctypes as C
import subprocess
import time

import pytest

from paper_2510_01565_b200 import binding as B
from paper_2510_01565_b200 import build


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return B.load_library()


def args(q_lens, kv_lens, heads, kv_heads, dim=64):
    n = len(q_lens)
    a = B.DitPromptAttentionArgs()
    a.type, a.n_heads, a.n_kv_heads, a.head_dim, a.causal, a.n_requests = 1, heads, kv_heads, dim, 1, n
    a.q_lens, a.kv_lens = (C.c_int32 * n)(*q_lens), (C.c_int32 * n)(*kv_lens)
    return a


MIXED = [1 + 97 * i % 300 for i in range(63)]


@pytest.mark.parametrize("q_lens,kv_lens,heads,kv_heads", [([8192], [8192], 4, 4), ([16384], [16384], 1, 1), (MIXED + [4000], MIXED + [12000], 4, 4),
                                                           ([256], [1000000], 32, 2), ([256], [100000000], 32, 2)])
def test_a_cut_batch_is_laid_out_in_little_time(lib, q_lens, kv_lens, heads, kv_heads):
    """The least of many runs, in us.  (What a cut saves on the GPU begins at some 10 us.)"""
    a = args(q_lens, kv_lens, heads, kv_heads)
    assert lib.dit_prompt_attention_workspace(C.byref(a)) > 0                     # (it is cut, or a few rows in parts)
    least = float("inf")
    for _ in range(300):
        start = time.perf_counter()
        lib.dit_prompt_attention_workspace(C.byref(a))
        least = min(least, 1e6 * (time.perf_counter() - start))
        if least < 25.0:
            break
    assert least < 25.0


def test_a_call_from_python_lays_its_batch_out_once(lib):
    """The size of the workspace and the launch come from one plan: the binding does not ask for the size by itself."""
    wanted = subprocess.run(["nm", "-D", "--undefined-only", build.MARSHAL], capture_output=True, text=True, check=True).stdout
    assert "prompt_attention_in" in wanted and "dit_prompt_attention_workspace" not in wanted

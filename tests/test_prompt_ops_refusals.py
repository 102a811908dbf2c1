"""Argument errors of the 4-bit operators, rotary positions and attention over packed prompts (include/dit_ops.h): found on the host, before any
device is touched, so they are checked here without a GPU.  The pointers below are never followed."""
import ctypes as C

import pytest

from paper_2510_01565_b200 import binding as B
from paper_2510_01565_b200 import build

P = 1 << 20          # an aligned address that nothing reads
OK, INVALID, SHAPE, CAPACITY = 0, 1, 2, 3
BIG = 2 ** 31
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return B.load_library()


def test_scale_bytes(lib):
    size = lib.dit_fp4_scale_bytes
    assert size(1, 1, 16) == 512 and size(128, 64, 16) == 512 and size(129, 65, 16) == 2048 and size(129, 128, 32) == 1024 and size(128, 129, 32) == 1024
    assert size(0, 5, 16) == 0 and size(5, 0, 16) == 0 and size(-1, 5, 16) == 0 and size(5, 5, 64) == 0 and size(BIG, 1, 16) == 0


@pytest.mark.parametrize("weight", [False, True])
def test_quantiser_refusals(lib, weight):
    def call(**kw):
        a = dict(x=P, type=1, ld=384, a=256, b=384, group=16, codes=P, ldc=192, scales=P, rows=P)
        a.update(kw)
        return (lib.dit_quantize_weight_fp4 if weight else lib.dit_quantize_fp4)(
            a["x"], a["type"], a["ld"], a["a"], a["b"], a["group"], a["codes"], a["ldc"], a["scales"], a["rows"], None)
    bad = [dict(x=None), dict(codes=None), dict(scales=None), dict(rows=None), dict(type=3), dict(type=-1), dict(group=8), dict(group=0), dict(ld=383),
           dict(ldc=200), dict(ldc=-192), dict(x=P + 1), dict(codes=P + 8), dict(scales=P + 8), dict(rows=P + 2), dict(type=2, x=P + 2), dict(group=32)]
    bad += [dict(ldc=112)] if weight else [dict(ldc=176), dict(a=-1)]
    for kw in bad:                                       # (group 32 has no row scales: a pointer to some is refused)
        assert call(**kw) == INVALID, kw
    for kw in (dict(a=2 ** 30 + 1, ld=2 ** 31, ldc=2 ** 30) if weight else dict(b=2 ** 30 + 1, ld=2 ** 31, ldc=2 ** 30), dict(a=BIG), dict(b=BIG), dict(a=2 ** 30, b=2 ** 30, ld=2 ** 30, ldc=2 ** 30), dict(b=0), dict(b=-3)) + ((dict(a=0),) if weight else ()):
        assert call(**kw) == SHAPE, kw
    if not weight:
        assert call(a=0) == OK and call(a=0, x=None, codes=None) == OK and call(a=0, group=7) == INVALID


def test_dequantiser_refusals(lib):
    def call(**kw):
        a = dict(codes=P, ldc=192, scales=P, rows=P, m=10, n=384, group=16, out=P, type=0, ld=384)
        a.update(kw)
        return lib.dit_dequantize_fp4(*a.values(), None)
    for kw in (dict(codes=None), dict(scales=None), dict(out=None), dict(type=5), dict(group=17), dict(m=-1), dict(ldc=176), dict(ldc=196), dict(ld=383), dict(codes=P + 1),
               dict(scales=P + 4), dict(rows=P + 1), dict(out=P + 1), dict(type=2, out=P + 2)):
        assert call(**kw) == INVALID, kw
    for kw in (dict(n=0), dict(m=BIG), dict(n=BIG)):
        assert call(**kw) == SHAPE, kw
    assert call(m=0, codes=None, out=None) == OK


def test_product_refusals(lib):
    def call(**kw):
        a = dict(a=P, a_scales=P, a_rows=P, b=P, b_scales=P, b_rows=P, bias=None, out=P, lda=128, ldb=128, ld_out=64, m=32, n=64, k=256, group=16, type=0)
        a.update(kw)
        return lib.dit_gemm_fp4(C.byref(B.DitGemmFp4Args(*a.values())), None)
    for name in ("a", "a_scales", "b", "b_scales", "out"):
        assert call(**{name: None}) == INVALID, name
    for kw in (dict(type=3), dict(group=4), dict(m=-1), dict(lda=112), dict(lda=136), dict(ldb=120), dict(ld_out=63), dict(a=P + 8), dict(b=P + 1), dict(a_scales=P + 8),
               dict(b_scales=P + 1), dict(a_rows=P + 1), dict(b_rows=P + 2), dict(bias=P + 2), dict(out=P + 1), dict(out=P + 2, type=2)):
        assert call(**kw) == INVALID, kw
    for kw in (dict(n=0), dict(k=0), dict(n=-3), dict(m=BIG), dict(n=2 ** 30 + 1), dict(k=2 ** 30 + 1), dict(m=2 ** 30, n=2 ** 30, ld_out=2 ** 30)):
        assert call(**kw) == SHAPE, kw
    assert call(m=0, a=None, out=None) == OK
    assert lib.dit_gemm_fp4(None, None) == INVALID


def lens(*x):
    return (C.c_int32 * len(x))(*x)


def test_rotary_refusals(lib):
    def call(**kw):
        a = dict(x=P, out=2 * P, ld_x=512, ld_out=512, rows=7, type=0, heads=4, dim=128, rotary=64, interleaved=0, inverse=0, base=10000.0, factor=2.0, trained=0.0, low=0.0,
                 high=0.0, magnitude=1.0, positions=None, n=2, lens=lens(3, 4), first=lens(0, 9))
        a.update(kw)
        return lib.dit_rotary(C.byref(B.DitRotaryArgs(*a.values())), None)
    none = C.POINTER(C.c_int32)()
    for kw in (dict(x=None), dict(out=None), dict(type=4), dict(rows=-1), dict(heads=0), dict(ld_x=511), dict(ld_out=100), dict(x=P + 1), dict(out=P + 1), dict(type=2, x=P + 2),
               dict(base=0.0), dict(base=-1.0), dict(base=NAN), dict(base=INF), dict(factor=0.5), dict(factor=NAN), dict(factor=INF), dict(trained=-1.0), dict(trained=NAN),
               dict(trained=100.0, low=2.0, high=2.0), dict(trained=100.0, low=1.0, high=INF), dict(trained=100.0, low=NAN, high=2.0), dict(magnitude=NAN), dict(rows=8), dict(lens=none),
               dict(n=-1), dict(lens=lens(3, -4)), dict(first=lens(0, -1)), dict(positions=P + 2), dict(out=P, ld_out=520)):
        assert call(**kw) == INVALID, kw
    for kw in (dict(rows=BIG), dict(dim=4097), dict(dim=1), dict(rotary=0), dict(rotary=63), dict(rotary=130), dict(dim=512, rotary=258), dict(heads=2 ** 20), dict(first=lens(0, 2 ** 31 - 4)),
               dict(lens=lens(2 ** 31 - 1, 2 ** 31 - 1))):
        assert call(**kw) == SHAPE, kw
    assert call(n=65, lens=lens(*[0] * 65), first=none, rows=0) == CAPACITY
    assert call(rows=0, n=0, lens=none, first=none, x=None) == OK and call(rows=0, n=2, lens=lens(0, 0), first=none) == OK and call(rows=0, positions=P) == OK
    assert lib.dit_rotary(None, None) == INVALID


def test_attention_refusals(lib):
    def args(**kw):
        a = dict(q=P, k=P, v=P, out=P, ld_q=512, ld_k=256, ld_v=256, ld_out=512, type=0, heads=4, kv_heads=2, dim=128, causal=1, scale=0.0, n=2, q_lens=lens(3, 4), kv_lens=lens(3, 9),
                 workspace=None, size=0)
        a.update(kw)
        return B.DitPromptAttentionArgs(*a.values())
    call = lambda **kw: lib.dit_prompt_attention(C.byref(args(**kw)), None)
    none = C.POINTER(C.c_int32)()
    for kw in (dict(q=None), dict(k=None), dict(v=None), dict(out=None), dict(type=2), dict(heads=0), dict(kv_heads=0), dict(kv_heads=3), dict(ld_q=504), dict(ld_q=516), dict(ld_k=255),
               dict(ld_v=250), dict(ld_out=511), dict(q=P + 8), dict(k=P + 2), dict(v=P + 4), dict(out=P + 8), dict(scale=-1.0), dict(scale=NAN), dict(scale=3e38), dict(n=-1), dict(q_lens=none),
               dict(kv_lens=none), dict(q_lens=lens(-1, 3)), dict(kv_lens=lens(3, -9))):
        assert call(**kw) == INVALID, kw
    for kw in (dict(dim=96), dict(dim=0), dict(heads=2 ** 14, kv_heads=1), dict(q_lens=lens(2 ** 31 - 1, 5)), dict(kv_lens=lens(2 ** 31 - 1, 2 ** 31 - 1))):
        assert call(**kw) == SHAPE, kw
    assert call(n=65, q_lens=lens(*[0] * 65), kv_lens=lens(*[0] * 65)) == CAPACITY
    assert call(q_lens=lens(0, 0), q=None, out=None) == OK and call(n=0, q_lens=none, kv_lens=none) == OK
    assert lib.dit_prompt_attention(None, None) == INVALID
    # single rows against long contexts are joined from parts, which need room
    long = dict(q_lens=lens(1, 2), kv_lens=lens(9000, 500))
    need = lib.dit_prompt_attention_workspace(C.byref(args(**long)))
    assert need > 0 and need % 16 == 0
    assert call(**long) == INVALID and call(**long, workspace=P + 8, size=need) == INVALID and call(**long, workspace=P, size=need - 1) == CAPACITY
    assert lib.dit_prompt_attention_workspace(C.byref(args())) == 0 and lib.dit_prompt_attention_workspace(C.byref(args(dim=80))) == 0
    assert lib.dit_prompt_attention_workspace(None) == 0


def test_workspace_does_not_depend_on_pointers_and_stays_small(lib):
    """One row or a few, any number of requests: the parts of the whole device, not of the contexts."""
    for n, q, kv in ((1, 1, 1_000_000), (64, 1, 30_000), (64, 16, 100), (3, 40, 70_000)):
        a = B.DitPromptAttentionArgs(None, None, None, None, 0, 0, 0, 0, 1, 32, 8, 128, 1, 0.0, n, lens(*[q] * n), lens(*[kv] * n), None, 0)
        assert lib.dit_prompt_attention_workspace(C.byref(a)) <= 64 << 20


def test_binding_refuses_what_it_cannot_describe():
    import torch
    x = torch.zeros(4, 256, dtype=torch.float16)
    for f in (lambda: B.dit_quantize_fp4(x), lambda: B.dit_quantize_weight_fp4(x), lambda: B.dit_dequantize_fp4(x, x, 4), lambda: B.dit_gemm_fp4(x, x, x, x, 4),
              lambda: B.dit_rotary(x, 2, [4]), lambda: B.dit_prompt_attention(x, x, x, [4], [4], 2), lambda: B.dit_quantize_fp4(None), lambda: B.dit_rotary(None, 2, [4])):
        with pytest.raises(B.DitError) as e:
            f()                                          # not CUDA tensors
        assert e.value.status == INVALID

"""Argument errors of the context-free operators (include/dit_ops.h): found on the host, before any device is touched, so they
are checked here without a GPU.  The pointers below are never followed."""
import ctypes as C
import os
import re

import pytest

from paper_2510_01565_b200 import binding as B
from paper_2510_01565_b200 import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 20          # an aligned address that nothing reads
OK, INVALID, SHAPE = 0, 1, 2
BIG = 2 ** 31


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return B.load_library()


def test_every_declared_operator_is_exported(lib):
    header = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "dit_ops.h")).read(), flags=re.S)
    declared = set(re.findall(r"\b(dit_[a-z_0-9]+)\s*\(", header))
    assert declared == set(B.OPS_EXPORTS)
    for name in declared:
        assert hasattr(lib, name)


def test_quantize_refusals(lib):
    def call(**kw):
        a = dict(x=P, type=0, ld=256, rows=4, cols=256, codes=P, ldc=256, scales=P, lds=4)
        a.update(kw)
        return lib.dit_quantize_block128(a["x"], a["type"], a["ld"], a["rows"], a["cols"], a["codes"], a["ldc"], a["scales"], a["lds"], None)
    for kw in (dict(x=None), dict(codes=None), dict(scales=None), dict(type=3), dict(type=-1), dict(rows=-1), dict(ld=255), dict(ldc=255),
               dict(ldc=264), dict(ldc=240), dict(lds=3), dict(x=P + 1), dict(codes=P + 8), dict(scales=P + 2), dict(type=2, x=P + 2)):
        assert call(**kw) == INVALID, kw
    for kw in (dict(cols=0), dict(cols=-1), dict(rows=BIG), dict(cols=BIG)):
        assert call(**kw) == SHAPE, kw
    assert call(rows=0) == OK and call(rows=0, x=None, codes=None, scales=None) == OK

    def weight(**kw):
        a = dict(w=P, type=1, ld=384, n_in=256, n_out=384, codes=P, ldc=256, scales=P)
        a.update(kw)
        return lib.dit_quantize_weight_block128(a["w"], a["type"], a["ld"], a["n_in"], a["n_out"], a["codes"], a["ldc"], a["scales"], None)
    for kw in (dict(w=None), dict(codes=None), dict(scales=None), dict(type=7), dict(ld=383), dict(ldc=255), dict(ldc=250), dict(w=P + 1),
               dict(codes=P + 4), dict(scales=P + 1)):
        assert weight(**kw) == INVALID, kw
    for kw in (dict(n_in=0), dict(n_out=0), dict(n_in=-5), dict(n_out=BIG), dict(n_in=BIG), dict(n_in=2 ** 30, n_out=2 ** 30)):
        assert weight(**kw) == SHAPE, kw


def test_product_refusals(lib):
    def call(**kw):
        a = dict(a=P, a_scales=P, b=P, b_scales=P, bias=None, out=P, lda=256, ld_a_scales=32, ldb=256, ld_out=64, m=32, n=64, k=256, out_type=0)
        a.update(kw)
        return lib.dit_gemm_block128(C.byref(B.DitGemmBlock128Args(*a.values())), None)
    for name in ("a", "a_scales", "b", "b_scales", "out"):
        assert call(**{name: None}) == INVALID, name
    for kw in (dict(out_type=3), dict(m=-1), dict(lda=255), dict(lda=264), dict(ldb=248), dict(ld_a_scales=31), dict(ld_out=63), dict(a=P + 8),
               dict(b=P + 1), dict(a_scales=P + 2), dict(b_scales=P + 1), dict(bias=P + 2), dict(out=P + 1), dict(out=P + 2, out_type=2)):
        assert call(**kw) == INVALID, kw
    for kw in (dict(n=0), dict(k=0), dict(n=-3), dict(m=BIG), dict(n=BIG), dict(k=BIG), dict(m=2 ** 30, n=2 ** 30, ld_a_scales=2 ** 30, ld_out=2 ** 30)):
        assert call(**kw) == SHAPE, kw
    assert call(m=0, a=None, out=None) == OK
    assert lib.dit_gemm_block128(None, None) == INVALID


def test_binding_refuses_what_it_cannot_describe():
    import torch
    x = torch.zeros(4, 256, dtype=torch.float16)
    with pytest.raises(B.DitError) as e:
        B.dit_quantize_block128(x)                      # not a CUDA tensor
    assert e.value.status == INVALID
    with pytest.raises(B.DitError):
        B.dit_gemm_block128(x, x, x, x)


def batch(**kw):
    """(struct, the arrays it points to): two requests, two heads of 64."""
    a = dict(q=P, k=P, v=P, ld_q=128, ld_k=128, ld_v=128, type=0, n_heads=2, head_dim=64, q_lens=[200, 1], kv_lens=[300, 40])
    a.update(kw)
    n = a.pop("n", len(a["q_lens"] or a["kv_lens"] or []))
    lens = [None if a[x] is None else (C.c_int32 * max(1, len(a[x])))(*a[x]) for x in ("q_lens", "kv_lens")]
    return B.DitAttentionBatch(*[a[x] for x in ("q", "k", "v", "ld_q", "ld_k", "ld_v", "type", "n_heads", "head_dim")], n, *lens), lens


BAD_BATCHES = [(dict(q=None), INVALID), (dict(k=None), INVALID), (dict(type=2), INVALID), (dict(type=-1), INVALID), (dict(n_heads=0), INVALID), (dict(n=-1), INVALID),
               (dict(ld_q=120), INVALID), (dict(ld_k=132), INVALID), (dict(q=P + 8), INVALID), (dict(k=P + 2), INVALID), (dict(q_lens=[-1, 5]), INVALID),
               (dict(kv_lens=[4, -1]), INVALID), (dict(q_lens=None, n=2), INVALID), (dict(kv_lens=None, n=2), INVALID), (dict(head_dim=96, ld_q=192, ld_k=192), SHAPE),
               (dict(head_dim=32), SHAPE), (dict(kv_lens=[128 * 16384 + 1, 1]), SHAPE), (dict(q_lens=[2 ** 31 - 1, 2 ** 31 - 1]), SHAPE), (dict(n=65), 3)]


@pytest.mark.parametrize("kw,status", BAD_BATCHES)
def test_attention_batches_refused_by_both_operators(lib, kw, status):
    b, _keep = batch(**kw)
    two = (C.c_int32 * 2)(1, 1)
    assert lib.dit_select_blocks(C.byref(b), two, None, P, P, 4, P, 1 << 30, None) == status
    assert lib.dit_block_attention(C.byref(b), P, P, 4, 0.0, P, 128, None) == status
    if "q" not in kw and "k" not in kw and "ld_q" not in kw and "ld_k" not in kw:
        assert lib.dit_select_blocks_workspace(C.byref(b)) == 0


def test_selector_refusals(lib):
    b, _keep = batch()
    size = lib.dit_select_blocks_workspace(C.byref(b))
    assert size == (3 + 4) * 128 * 8 and lib.dit_select_blocks_workspace(None) == 0
    ints = lambda *x: (C.c_int32 * len(x))(*x)

    def call(keep=ints(2, 1), tail=None, index=P, count=P, ld=2, ws=P, nbytes=size):
        return lib.dit_select_blocks(C.byref(b), keep, tail, index, count, ld, ws, nbytes, None)
    for kw in (dict(keep=None), dict(keep=ints(0, 1)), dict(keep=ints(2, -1)), dict(tail=ints(-1, 0)), dict(index=None), dict(count=None), dict(ld=1),
               dict(ws=None), dict(ws=P + 8), dict(index=P + 2)):
        assert call(**kw) == INVALID, kw
    assert call(nbytes=size - 1) == 3
    empty, _e = batch(q_lens=[0, 0])
    assert lib.dit_select_blocks(C.byref(empty), None, None, None, None, 0, None, 0, None) == OK
    assert lib.dit_select_blocks(None, None, None, None, None, 0, None, 0, None) == INVALID


def test_attention_refusals(lib):
    b, _keep = batch()

    def call(batch_=b, index=P, count=P, ld=2, scale=0.0, out=P, ld_out=128):
        return lib.dit_block_attention(C.byref(batch_), index, count, ld, scale, out, ld_out, None)
    for kw in (dict(index=None), dict(count=None), dict(out=None), dict(ld=0), dict(ld_out=120), dict(ld_out=129), dict(out=P + 8), dict(index=P + 1),
               dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf"))):
        assert call(**kw) == INVALID, kw
    for kw in (dict(v=None), dict(ld_v=100), dict(ld_v=100, v=P), dict(v=P + 4)):
        bad, _k = batch(**kw)
        assert call(bad) == INVALID, kw
    empty, _e = batch(q_lens=[0, 0])
    assert call(empty, index=None, out=None) == OK
    assert lib.dit_block_attention(None, P, P, 2, 0.0, P, 128, None) == INVALID


def test_workspace_of_the_reduced_modes(lib):
    def ws(**kw):
        base = dict(hidden=384, n_heads=6, head_dim=64, mlp_hidden=1536, cond_dim=384, max_blocks=2, max_total_tokens=1000, max_requests=3, ln_eps=1e-6, flags=0)
        base.update(kw)
        return lib.dit_workspace_bytes(C.byref(B.DitConfig(*base.values())))
    full, slack = ws(), 8 * 1024
    # the quantised operand [T, H + F] and its scales [(H + F) / 128, T]
    need = 1000 * (384 + 1536) + 15 * 1000 * 4
    assert need <= ws(flags=B.DIT_FLAG_FP8_BLOCK128) - full <= need + slack
    # means of at most T / 128 + requests query and key blocks in 64 bits, lists of at most ceil(T / 128) entries
    blocks = 1000 // 128 + 3
    need = 2 * blocks * 384 * 8 + 6 * blocks * 8 * 4 + 6 * blocks * 4
    assert need <= ws(flags=B.DIT_FLAG_SPARSE_ATTENTION) - full <= need + slack
    assert ws(flags=B.DIT_FLAG_SPARSE_ATTENTION | 8) > 0 and ws(flags=B.DIT_FLAG_SPARSE_ATTENTION | 7) > 0
    # a very wide MLP has more 128 x 128 blocks than output channels
    wide = dict(hidden=64, n_heads=1, mlp_hidden=64 * 300)
    assert ws(flags=B.DIT_FLAG_FP8_BLOCK128, **wide) > ws(**wide)
    for bad in (16, 32 | 1, 32 | 2, 32 | 4, 32 | 8, 128):
        assert ws(flags=bad) == 0, bad
    assert lib.dit_ctx_set_sparse_attention(None, 0.5, 1) == INVALID


def test_a_scale_whose_product_with_log2_e_is_infinite_is_refused(lib):
    b, keepalive = B.DitAttentionBatch(), (C.c_int32 * 1)(4)
    for name, value in dict(q=P, k=P, v=P, ld_q=128, ld_k=128, ld_v=128, type=0, n_heads=1, head_dim=128, n_requests=1, q_lens=keepalive, kv_lens=keepalive).items():
        setattr(b, name, value)
    for scale in (2.4e38, 3.0e38):
        assert lib.dit_block_attention(C.byref(b), P, P, 1, scale, P, 128, None) == INVALID


def test_the_steps_gelu_product_refuses_rows_off_16_byte_boundaries(lib):
    """The library's own launcher (C++, no entry point reaches it with such an output): before, the kernel for many rows would have stored
    the values in front of the GELU there.  The refusal comes before the device is looked at, without which this machine has another error
    to report; the product has no rows, so that nothing could run where there is a device."""
    class Product(C.Structure):
        _fields_ = ([(n, C.c_void_p) for n in ("a", "a_scales", "b", "b_scales", "bias", "out")] + [(n, C.c_longlong) for n in ("lda", "ld_a_scales", "ldb", "ld_out")]
                    + [(n, C.c_int) for n in ("m", "n", "k", "plan_m", "epilogue", "row0")] + [("resid", C.c_void_p), ("gate", C.c_void_p), ("gate_stride", C.c_longlong),
                                                                                               ("status", C.c_void_p)])
    launch = lib["_ZN3dit20launch_block_productERKNS_12BlockProductERKNS_7SeqInfoEP11CUstream_st"]
    launch.restype, launch.argtypes = C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p]
    seq = C.create_string_buffer(1 << 16)
    gelu, invalid_value = 3, 1

    def call(out, ld_out):
        b = Product(P, P, P, P, None, out, 128, 4096, 128, ld_out, 0, 4096, 128, 4096, gelu, 0, None, None, 0, None)
        return launch(C.byref(b), C.cast(seq, C.c_void_p), None)
    for out, ld_out in ((P + 2, 4096), (P + 8, 4096), (P, 4097), (P, 4100)):
        assert call(out, ld_out) == invalid_value


def test_binding_refuses_lazily_negated_views():
    """The imaginary part of a conjugate has its sign in a flag of the tensor, not in its memory."""
    import torch
    x = torch.randn(40, 1, dtype=torch.complex64).conj().imag
    assert x.is_neg()
    for call in (lambda: B.dit_quantize_block128(x), lambda: B.dit_quantize_weight_block128(x), lambda: B.dit_select_blocks(x, x, [40], [40], 1, [1])):
        with pytest.raises(B.DitError, match="negated") as e:
            call()
        assert e.value.status == INVALID

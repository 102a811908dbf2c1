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

"""The 4-bit quantisers, the values that their results stand for, and the product, against plain evaluations.

Codes, scale bytes and row scales are functions of single fp32 operations: compared bit for bit.  The product is compared with its definition in
64 bits; how far it may be off is counted from the arithmetic:
  * the tensor cores add k exact products of two 2-bit significands and two scales in fp32 in some order, each addition off by at most one
    unit in the last place of the running sum (2^-23 relative, whether it rounds or cuts off): k * 2^-23 * sum|a b|; up to eight joined
    partial sums: 8 * 2^-24 more;
  * row scale, column scale and bias: three roundings, 3 * 2^-24 of the result's parts;
  * a 16-bit output is rounded once: half a step, or half the smallest subnormal.
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


def draw(seed, rows, cols, dtype):
    """Rows of very different size, a few loud columns, some columns of zeros."""
    import torch
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g) * torch.exp(torch.randn(rows, 1, generator=g))
    x = torch.where(torch.rand(cols, generator=g) < 0.02, 30.0 * x, x)
    return torch.where(torch.rand(rows, (cols + 15) // 16, generator=g).repeat_interleave(16, 1)[:, :cols] < 0.05, 0.0, x).to(dtype)


def check_quantised(got, x, group):
    """x: the quantised matrix as fp64 [rows, columns]."""
    codes, scales, row_scales = got
    want = P.quantize(x, group)
    assert np.array_equal(codes.cpu().numpy(), P.pack(want[0]))
    assert np.array_equal(scales.cpu().numpy(), P.scale_tiles(want[1], group))
    if group == 16:
        assert np.array_equal(row_scales.cpu().numpy().astype(np.float64), want[2])
    else:
        assert row_scales is None
    return want


SHAPES = [(1, 1), (1, 16), (1, 384), (3, 31), (9, 33), (33, 129), (77, 1000), (130, 260), (129, 1537), (300, 4100), (5, 20000)]


@pytest.mark.parametrize("group", [16, 32])
@pytest.mark.parametrize("kind", ["float16", "bfloat16", "float32"])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_quantize_rows_bit_for_bit(B, rows, cols, kind, group):
    import torch
    x = draw(rows + cols, rows, cols, getattr(torch, kind))
    got = B.dit_quantize_fp4(x.cuda(), group)
    want = check_quantised(got, x.double().numpy(), group)
    for out in (torch.float32, torch.float16, torch.bfloat16):
        v = B.dit_dequantize_fp4(got[0], got[1], cols, group, got[2], out_dtype=out)
        exact = torch.from_numpy(P.values(*want, group))
        limit = torch.finfo(out).max
        assert torch.equal(v.cpu(), exact.float().clamp(-limit, limit).to(out))       # (the values have six bits: fp32 holds them)


@pytest.mark.parametrize("group", [16, 32])
@pytest.mark.parametrize("kind", ["float16", "bfloat16", "float32"])
@pytest.mark.parametrize("n_in,n_out", [(1, 1), (33, 7), (128, 64), (200, 130), (1000, 77), (257, 1024), (2049, 65)])
def test_quantize_weight_bit_for_bit(B, n_in, n_out, kind, group):
    import torch
    w = 0.02 * draw(n_in + n_out, n_in, n_out, getattr(torch, kind))
    check_quantised(B.dit_quantize_weight_fp4(w.cuda(), group), w.t().double().numpy(), group)


@pytest.mark.parametrize("group", [16, 32])
def test_borders_of_codes_and_scales(B, group):
    """Every border between two codes, exactly on it and one step of the type to either side; maxima at the scale's limits."""
    import torch
    for kind in (torch.float16, torch.bfloat16, torch.float32):
        border = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
        near = torch.cat([border, border * (1 + 2 * torch.finfo(kind).eps), border * (1 - torch.finfo(kind).eps)])
        rows = []
        for top in (6.0, 6.0 * (1 + torch.finfo(kind).eps), 4.0, 3.0, 5.5):
            for s in (1.0, 1.125, 1.875, 2.0 ** -9, 3.5):
                rows.append(torch.cat([torch.tensor([top]), near, -near, torch.zeros(21)]).roll(len(rows)) * s)
        x = torch.stack(rows).to(kind)
        if group == 16:
            x[:, 0] = 6 * 448 * 2.0 ** -5         # a loud first group fixes the row's factor
        check_quantised(B.dit_quantize_fp4(x.cuda(), group), x.double().numpy(), group)


@pytest.mark.parametrize("group", [16, 32])
def test_extreme_magnitudes(B, group):
    import torch
    x = torch.zeros(8, 96)
    x[0, 3], x[1, 3], x[2, 3] = 3.3e38, 1e-38, 2.0 ** -149
    x[3] = 2.0 ** -100 * torch.arange(96)
    x[4] = torch.finfo(torch.float32).max
    x[5, ::7], x[5, 40] = 1e-6, 1e6
    x[6] = -0.0
    check_quantised(B.dit_quantize_fp4(x.cuda(), group), x.double().numpy(), group)


@pytest.mark.parametrize("kind", ["float16", "float32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("group", [16, 32])
def test_values_that_are_no_numbers_spoil_their_row_or_group_only(B, group, bad, kind):
    import torch
    x = draw(1, 40, 200, getattr(torch, kind))
    clean = B.dit_quantize_fp4(x.cuda(), group)
    y = x.clone()
    y[7, 70] = bad
    for got, ref in ((B.dit_quantize_fp4(y.cuda(), group), clean), (B.dit_quantize_weight_fp4(y.t().contiguous().cuda(), group), clean)):
        v = B.dit_dequantize_fp4(got[0], got[1], 200, group, got[2], out_dtype=torch.float32)
        w = B.dit_dequantize_fp4(ref[0], ref[1], 200, group, ref[2], out_dtype=torch.float32)
        spoilt = torch.zeros(40, 200, dtype=torch.bool)
        spoilt[7, 64:96 if group == 32 else 64] = True
        if group == 16:
            spoilt[7] = True
        assert v.isnan().cpu().equal(spoilt) and torch.equal(v.cpu()[~spoilt], w.cpu()[~spoilt])
        b = B.dit_quantize_fp4(torch.ones(130, 200, device="cuda"), group)
        out = B.dit_gemm_fp4(got[0], got[1], b[0], b[1], 200, group, got[2], b[2], out_dtype=torch.float32)
        assert out[7].isnan().all() and not out[torch.arange(40) != 7].isnan().any()


def test_strides_and_untouched_surroundings(B):
    import torch
    for kind in (torch.float16, torch.float32):
        big = draw(5, 70, 400, kind).cuda()
        for x in (big[:, 8:308], big[:, 3:302], big[1:66:2, 16:272]):
            rows, cols = x.shape
            half = (cols + 1) // 2
            codes = torch.full((rows + 2, 256), 0xAB, dtype=torch.uint8, device="cuda")
            got = B.dit_quantize_fp4(x, 16, codes=codes[1:-1, :half])
            check_quantised(got, x.double().cpu().numpy(), 16)
            assert (codes[0] == 0xAB).all() and (codes[-1] == 0xAB).all() and (codes[:, half:] == 0xAB).all()
            out = torch.full((rows + 2, 407), 9.0, dtype=kind, device="cuda")
            B.dit_dequantize_fp4(got[0], got[1], cols, 16, got[2], out=out[1:-1, 3:3 + cols])
            assert (out[0] == 9).all() and (out[-1] == 9).all() and (out[:, :3] == 9).all() and (out[:, 3 + cols:] == 9).all()


# ------------------------------------------------------------------------------------------------ product
def operand(seed, rows, k, group):
    import torch
    x = draw(seed, rows, k, torch.float32).cuda()
    return x


def check_product(B, m, n, k, group, out_dtype, bias, seed=0, **kw):
    import torch
    a = B.dit_quantize_fp4(draw(seed, m, k, torch.float32).cuda(), group)
    b = B.dit_quantize_fp4(0.02 * draw(seed + 1, n, k, torch.float32).cuda(), group)
    c = torch.randn(n, generator=torch.Generator().manual_seed(seed)).cuda() if bias else None
    got = B.dit_gemm_fp4(a[0], a[1], b[0], b[1], k, group, a[2], b[2], bias=c, out_dtype=out_dtype, **kw)
    va = B.dit_dequantize_fp4(a[0], a[1], k, group, a[2], out_dtype=torch.float32).double()
    vb = B.dit_dequantize_fp4(b[0], b[1], k, group, b[2], out_dtype=torch.float32).double()
    exact, size = va @ vb.t(), va.abs() @ vb.abs().t()
    tol = (k * 2.0 ** -23 + 8 * 2.0 ** -24 + 3 * 2.0 ** -24) * size
    if bias:
        exact = exact + c.double()
        tol = tol + 3 * 2.0 ** -24 * (exact.abs() + c.double().abs())
    info = torch.finfo(out_dtype)
    tol = tol + (exact.abs() + tol) * info.eps / 2 + info.smallest_normal * info.eps / 2
    exact = exact.clamp(-info.max, info.max)
    worst = ((got.double() - exact).abs() / tol).max().item()
    assert worst <= 1.0, worst
    return got


PRODUCTS = [(1, 1, 1), (1, 128, 64), (1, 1000, 2056), (2, 130, 33), (16, 257, 512), (17, 96, 700), (32, 500, 1000), (33, 640, 256), (77, 1000, 2056),
            (64, 128, 4096), (100, 300, 65), (129, 4001, 320), (200, 4096, 64), (256, 9216, 512), (700, 3000, 1024), (1000, 4104, 257), (300, 20000, 130),
            (2100, 2500, 768)]


@pytest.mark.parametrize("group", [16, 32])
@pytest.mark.parametrize("out", ["float16", "bfloat16", "float32"])
@pytest.mark.parametrize("m,n,k", PRODUCTS)
def test_product(B, m, n, k, out, group):
    import torch
    check_product(B, m, n, k, group, getattr(torch, out), bias=(m + n) % 2 == 0, seed=m + n + k)


@pytest.mark.parametrize("group", [16, 32])
def test_every_scale_reaches_its_own_group(B, group):
    """Codes of ones, one group after the other with a scale of its own: a product of two such operands names every pair of scales that met."""
    import torch
    for m, n, k in ((20, 300, 640), (130, 200, 640), (600, 2600, 640)):
        groups = -(-k // group)
        codes_a = torch.full((m, k // 2), 0x22, dtype=torch.uint8, device="cuda")
        codes_b = torch.full((n, k // 2), 0x22, dtype=torch.uint8, device="cuda")
        def scales(rows, seed):
            e = np.random.default_rng(seed).integers(-3, 4, (rows, groups))
            return np.exp2(e.astype(float))
        sa, sb = scales(m, 1), scales(n, 2)
        got = B.dit_gemm_fp4(codes_a, torch.from_numpy(P.scale_tiles(sa, group)).cuda(), codes_b, torch.from_numpy(P.scale_tiles(sb, group)).cuda(), k, group,
                             out_dtype=torch.float32)
        assert np.array_equal(got.double().cpu().numpy(), group * (sa @ sb.T))        # sums of powers of two: exact in fp32


def test_row_scales_of_any_size_and_infinite_sums(B):
    import torch
    a = B.dit_quantize_fp4(torch.ones(40, 256, device="cuda"), 16)
    b = B.dit_quantize_fp4(torch.ones(300, 256, device="cuda"), 16)
    ra, rb = a[2] * torch.logspace(-18, 18, 40, device="cuda"), b[2] * 3.0
    got = B.dit_gemm_fp4(a[0], a[1], b[0], b[1], 256, 16, ra, rb, out_dtype=torch.float32)
    one = 6 * 352 / 2048                          # what 1 becomes: row factor 2^-11, scale e4m3(2048 / 6) = 352, code 6
    want = 256 * 3.0 * one * one * torch.logspace(-18, 18, 40, device="cuda").double()
    assert ((got.double() - want[:, None]).abs() <= 4 * 2.0 ** -24 * want[:, None]).all()
    half = B.dit_gemm_fp4(a[0], a[1], b[0], b[1], 256, 16, ra, rb, out_dtype=torch.float16)
    assert (half[-1] == 65504).all()


def test_product_into_strided_memory(B):
    import torch
    for m, n, k in ((20, 300, 512), (600, 2600, 512)):
        for out_dtype in (torch.float16, torch.float32):
            for left, right in ((8, 8), (3, 2)):
                big = torch.full((m + 2, n + left + right), 5.0, dtype=out_dtype, device="cuda")
                view = big[1:-1, left:left + n]
                check_product(B, m, n, k, 16, out_dtype, True, out=view)
                assert (big[0] == 5).all() and (big[-1] == 5).all() and (big[:, :left] == 5).all() and (big[:, left + n:] == 5).all()


def test_rows_do_not_depend_on_the_batch(B):
    """A row's sum is taken in the order that the shapes of the call choose: the same call gives the same bits again."""
    import torch
    x = draw(3, 700, 1024, torch.float16).cuda()
    b = B.dit_quantize_weight_fp4(draw(4, 1024, 2000, torch.float16).cuda(), 16)
    a = B.dit_quantize_fp4(x, 16)
    first = B.dit_gemm_fp4(a[0], a[1], b[0], b[1], 1024, 16, a[2], b[2])
    for _ in range(3):
        assert torch.equal(first, B.dit_gemm_fp4(a[0], a[1], b[0], b[1], 1024, 16, a[2], b[2]))
    one = B.dit_quantize_fp4(x[5:6], 16)
    assert torch.equal(one[0][0], a[0][5]) and torch.equal(one[2][0], a[2][5])


def test_empty_batches(B):
    import torch
    x = torch.empty(0, 64, device="cuda")
    codes, scales, row_scales = B.dit_quantize_fp4(x, 16)
    assert codes.shape == (0, 32) and row_scales.shape == (0,)
    b = B.dit_quantize_fp4(torch.ones(8, 64, device="cuda"), 16)
    assert B.dit_gemm_fp4(codes, scales, b[0], b[1], 64, 16, row_scales, b[2]).shape == (0, 8)
    assert B.dit_dequantize_fp4(codes, scales, 64, 16, row_scales).shape == (0, 64)


@pytest.mark.parametrize("kind", ["float16", "float32"])
@pytest.mark.parametrize("group", [16, 32])
@pytest.mark.parametrize("cols", [1, 17, 40, 513, 1000, 6301, 13000, 26000])
def test_rows_that_start_on_other_boundaries_have_the_same_codes_and_values(B, cols, group, kind):
    """Starts on multiples of 32, 16, 8 and 4 bytes and of an element: each has its own loads and stores, and all give the oracle's bits."""
    import torch
    t = getattr(torch, kind)
    size, rows = t.itemsize, 37
    x = draw(cols, rows, cols, t)
    want = P.quantize(x.double().numpy(), group)
    values = P.values(*want, group)
    for start in (32, 16, 8, 4, size):
        pitch = (cols * size + 63) // 32 * 32 + start
        buffer = torch.full((rows, pitch // size), 9.0, dtype=t, device="cuda")
        part = buffer[:, start // size:start // size + cols]
        part.copy_(x)
        got = B.dit_quantize_fp4(part, group)
        check_quantised(got, x.double().numpy(), group)
        out = torch.full_like(buffer, 7.0)
        B.dit_dequantize_fp4(got[0], got[1], cols, group, got[2], out=out[:, start // size:start // size + cols])
        back = out.cpu()
        # (a value has six bits: rounding it to the type is the only one)
        inside = back[:, start // size:start // size + cols].double().numpy()
        assert np.array_equal(inside, torch.from_numpy(values).to(t).double().numpy())
        back[:, start // size:start // size + cols] = 7.0
        assert (back == 7.0).all()

"""Row factors of the 4-bit product and of the values, over all of fp32's range.

A factor that is a power of two changes no bit of a sum, so the product with factors is the product without them times both factors, rounded
once into the output's type: compared bit for bit, whatever the factors' sizes.  The result leaves the type's range where the whole product does, and not where a
part of it would.
"""
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


def operand(seed, rows, k, group, scale):
    """Codes at random under scales near 2^scale (groups of 32) or e4m3 numbers between 1/2 and 8 (groups of 16)."""
    import torch
    g = torch.Generator().manual_seed(seed)
    wide = ((k + 1) // 2 + 15) // 16 * 16
    codes = torch.randint(0, 256, (rows, wide), generator=g, dtype=torch.uint8).cuda()[:, :(k + 1) // 2]
    shape = ((rows + 127) // 128, -(-k // (4 * group)), 512)
    if group == 32:
        scales = torch.randint(scale + 126, scale + 129, shape, generator=g, dtype=torch.uint8)
    else:
        scales = torch.randint(0x30, 0x50, shape, generator=g, dtype=torch.uint8)
    return codes, scales.cuda()


# few rows; many, on 16-byte boundaries and off them
SIZES = [(5, 200, 512), (40, 300, 256), (2050, 1032, 256), (2050, 1027, 256)]
# of a row, of a column: their product is moderate, out of range, or below it
FACTORS = [2.0 ** 100, 2.0 ** -100, 1.0, 2.0 ** 120, 2.0 ** -120, 2.0 ** 60, 2.0 ** -126, 2.0 ** 127, 2.0 ** -3]


@pytest.mark.parametrize("kind", ["float16", "bfloat16", "float32"])
@pytest.mark.parametrize("group,scale", [(16, 0), (32, 0), (32, 50), (32, -50)])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_factors_of_opposite_size(B, m, n, k, group, scale, kind):
    import torch
    out_dtype = getattr(torch, kind)
    a, b = operand(m, m, k, group, scale), operand(n, n, k, group, scale)
    table = torch.tensor(FACTORS, device="cuda")
    ra, rb = table[torch.arange(m, device="cuda") % 9], table[torch.arange(n, device="cuda") % 7]
    rb = torch.where(torch.arange(n, device="cuda") % 11 == 3, -rb, rb)
    plain = B.dit_gemm_fp4(a[0], a[1], b[0], b[1], k, group, out_dtype=torch.float32).double()
    assert bool(plain.isfinite().all()) and bool((plain != 0).any())
    got = B.dit_gemm_fp4(a[0], a[1], b[0], b[1], k, group, a_row_scales=ra, b_row_scales=rb, out_dtype=out_dtype)
    want = (plain * ra.double()[:, None] * rb.double()).float()
    limit = torch.finfo(out_dtype).max
    if out_dtype != torch.float32:
        want = want.clamp(-limit, limit).to(out_dtype)
    # two factors below 1 may round twice where the result has left fp32's normal numbers: a step of the smallest number
    off = (got.double() - want.double()).abs()
    tiny = want.double().abs() < 2.0 ** -126
    same = (got == want) | (tiny & (off <= 2.0 ** -149))
    assert bool(same.all()), int((~same).sum())
    moderate = (ra.double()[:, None] * rb.double()).abs()
    assert int(((moderate > 2.0 ** -30) & (moderate < 2.0 ** 30)).sum()) * 6 > m * n           # (a good part of what is compared is moderate)
    B.dit_ops_poll_status()


@pytest.mark.parametrize("m,n,k", SIZES)
def test_factors_that_are_no_powers_of_two_and_a_bias(B, m, n, k):
    """Three roundings at most: of one product, of the next or of the factors', and of the sum with the bias."""
    import torch
    a, b = operand(1, m, k, 16, 0), operand(2, n, k, 16, 0)
    g = torch.Generator().manual_seed(m + n)
    large = torch.rand(m, generator=g) < 0.5
    ra = torch.where(large, 3.7e34, 2.3e-34) * (1 + torch.rand(m, generator=g))
    rb = torch.where(torch.rand(n, generator=g) < 0.5, 1.9e-34, 4.1e-1) * (1 + torch.rand(n, generator=g))
    bias = torch.randn(n, generator=g).cuda()
    ra, rb = ra.cuda(), rb.cuda()
    plain = B.dit_gemm_fp4(a[0], a[1], b[0], b[1], k, 16, out_dtype=torch.float32).double()
    got = B.dit_gemm_fp4(a[0], a[1], b[0], b[1], k, 16, a_row_scales=ra, b_row_scales=rb, bias=bias, out_dtype=torch.float32).double()
    part = plain * ra.double()[:, None] * rb.double()
    want = part + bias.double()
    fits = part.abs() < 2.0 ** 127
    room = 2 * 2.0 ** -24 * part.abs() * (1 + 2.0 ** -20) + 2.0 ** -24 * want.abs() * (1 + 2.0 ** -20) + 2.0 ** -148
    assert bool(((got - want).abs() <= room)[fits].all()) and int(fits.sum()) * 4 > m * n
    assert bool((got[~fits].abs() >= 2.0 ** 126).all())


@pytest.mark.parametrize("cols", [256, 250])
@pytest.mark.parametrize("kind", ["float16", "bfloat16", "float32"])
@pytest.mark.parametrize("group", [16, 32])
def test_values_of_large_scales_under_small_row_factors(B, group, kind, cols):
    import torch
    out_dtype = getattr(torch, kind)
    rows = 140
    codes = torch.randint(0, 256, (rows, 128), generator=torch.Generator().manual_seed(1), dtype=torch.uint8).cuda()[:, :(cols + 1) // 2]
    shape = (2, -(-cols // (4 * group)), 512)
    byte = torch.arange(512) % 128 if group == 16 else torch.arange(512) % 255
    byte = torch.where(byte == 127, 126, byte) if group == 16 else byte
    scales = byte.to(torch.uint8).expand(shape).contiguous().cuda()
    # (of the very large and the very small scales, a value under each factor lies inside fp32)
    factors = torch.tensor([1.0, 2.0 ** -100, 2.0 ** 100, 2.0 ** -20, -2.0 ** -126, 1.5, 2.0 ** 127], device="cuda")[torch.arange(rows, device="cuda") % 7]
    got = B.dit_dequantize_fp4(codes, scales, cols, group, factors, out_dtype=out_dtype)
    levels = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device="cuda")
    col, row = torch.arange(cols, device="cuda"), torch.arange(rows, device="cuda")[:, None]
    code = ((codes.int()[:, col // 2] >> (4 * (col % 2))) & 15).long()
    value = torch.where(code >= 8, -levels[code & 7], levels[code & 7])
    at = col // group
    byte = scales[row // 128, at // 4, row % 32 * 16 + row % 128 // 32 * 4 + at % 4]
    scale = byte.view(torch.float8_e4m3fn).double() if group == 16 else torch.exp2(byte.double() - 127.0)
    want = (value * scale * factors.double()[:, None]).float()
    if out_dtype != torch.float32:
        limit = torch.finfo(out_dtype).max
        want = want.clamp(-limit, limit).to(out_dtype)
    assert torch.equal(got, want)


def test_a_row_in_batches_of_other_sizes(B):
    """The same rows among 3, 60 and 2100: kernels and cuts of k differ, so their sums may, within what k additions in fp32 allow."""
    import torch
    k, n = 1000, 1100
    a, b = operand(7, 2100, k, 32, 0), operand(8, n, k, 32, 0)
    rows = [B.dit_gemm_fp4(a[0][:m], a[1][:(m + 127) // 128], b[0], b[1], k, 32, out_dtype=torch.float32)[:3].double() for m in (3, 60, 2100)]
    va, vb = (B.dit_dequantize_fp4(x[0][:r], x[1][:(r + 127) // 128], k, 32, out_dtype=torch.float32).double() for x, r in ((a, 3), (b, n)))
    room = (k + 8) * 2.0 ** -23 * (va.abs() @ vb.abs().t())
    for got in rows:
        assert bool(((got - va @ vb.t()).abs() <= room).all())

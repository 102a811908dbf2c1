"""The block-scaled e4m3 product and its quantisers against plain evaluations.

The quantiser is compared bit for bit with the same three fp32 operations done by torch on the CPU.  The product is
compared with its definition in 64 bits; how far it may be off is counted from the arithmetic:
  * inside a group the tensor core adds at most 128 exact products in fp32, each addition off by at most one unit in the last
    place of the running sum (2^-23 relative, whether it rounds or cuts off), so by 128 * 2^-23 * sum|a b|;
  * scaling (one rounding for sa * sb, one for the multiply-add) and adding G groups and the bias costs at most
    (G + 3) * 2^-24 of the sum of magnitudes; a joined split adds up to 8 partial sums: 8 * 2^-24 more;
  * a 16-bit output is rounded once: half a step, or half the smallest subnormal.
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


def plain_quantize(x, weight):
    """Codes (as fp32 values) and scales of a CPU matrix, by single fp32 operations."""
    import torch
    x = x.float().t() if weight else x.float()
    rows, cols = x.shape
    tall = 128 if weight else 1
    x = torch.nn.functional.pad(x, (0, -cols % 128, 0, -rows % tall))
    blocks = x.reshape(x.shape[0] // tall, tall, x.shape[1] // 128, 128)
    top = blocks.abs().amax(dim=(1, 3), keepdim=True)
    top = torch.where(top < 2.0 ** -100, torch.full_like(top, 2.0 ** -100), top)
    full = torch.full_like(top, 448.0)
    codes = (blocks * (full / top)).clamp(-448, 448).to(torch.float8_e4m3fn).float().reshape(x.shape)[:rows, :cols]
    scales = (top / full)[:, 0, :, 0]
    return codes, scales if weight else scales.t()


def draw(seed, rows, cols, dtype, spread=1.0):
    import torch
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g) * torch.exp(spread * torch.randn(rows, 1, generator=g))
    return x.to(dtype)


SHAPES = [(1, 1), (1, 384), (3, 127), (9, 128), (33, 129), (77, 1000), (130, 260), (300, 513), (5000, 640)]


@pytest.mark.parametrize("kind", ["float16", "bfloat16", "float32"])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_quantize_rows_bit_for_bit(B, rows, cols, kind):
    import torch
    x = draw(rows + cols, rows, cols, getattr(torch, kind))
    codes, scales = B.dit_quantize_block128(x.cuda())
    want_codes, want_scales = plain_quantize(x, False)
    assert torch.equal(codes.float().cpu(), want_codes) and torch.equal(scales.cpu(), want_scales)


@pytest.mark.parametrize("kind", ["float16", "bfloat16", "float32"])
@pytest.mark.parametrize("n_in,n_out", SHAPES + [(384, 1), (129, 33), (1000, 77), (260, 130)])
def test_quantize_weight_bit_for_bit(B, n_in, n_out, kind):
    import torch
    w = draw(n_in + 2 * n_out, n_in, n_out, getattr(torch, kind))
    codes, scales = B.dit_quantize_weight_block128(w.cuda())
    want_codes, want_scales = plain_quantize(w, True)
    assert torch.equal(codes.float().cpu(), want_codes) and torch.equal(scales.cpu(), want_scales)


@pytest.mark.parametrize("kind", ["float16", "bfloat16", "float32"])
def test_quantize_reads_strided_and_unaligned_rows_and_leaves_the_padding(B, kind):
    import torch
    x = draw(3, 37, 300, getattr(torch, kind)).cuda()
    for left, right in ((0, 4), (1, 2), (8, 8)):                       # the second starts off a 16-byte boundary
        wide = torch.zeros(37, left + 300 + right, dtype=x.dtype, device="cuda")
        view = wide[:, left:left + 300]
        view.copy_(x)
        buf = torch.full((39, 320), 0x33, dtype=torch.uint8, device="cuda")
        sbuf = torch.full((3, 64), -7.0, device="cuda")
        codes, scales = buf.view(torch.float8_e4m3fn)[1:38, :300], sbuf[:, :37]
        B.dit_quantize_block128(view, codes=codes, scales=scales)
        want_codes, want_scales = plain_quantize(x.cpu(), False)
        assert torch.equal(codes.float().cpu(), want_codes) and torch.equal(scales.cpu(), want_scales)
        assert bool((buf[:, 300:] == 0x33).all()) and bool((buf[0] == 0x33).all()) and bool((buf[38] == 0x33).all())
        assert bool((sbuf[:, 37:] == -7.0).all())
        cbuf = torch.full((302, 48), 0x33, dtype=torch.uint8, device="cuda")
        wcodes = cbuf.view(torch.float8_e4m3fn)[1:301, :37]
        _, wscales = B.dit_quantize_weight_block128(view, codes=wcodes)
        want_codes, want_scales = plain_quantize(x.cpu(), True)
        assert torch.equal(wcodes.float().cpu(), want_codes) and torch.equal(wscales.cpu(), want_scales)
        assert bool((cbuf[:, 37:] == 0x33).all()) and bool((cbuf[0] == 0x33).all()) and bool((cbuf[301] == 0x33).all())


def test_quantize_zeros_tiny_huge_and_non_finite_groups(B):
    import torch
    x = torch.zeros(6, 256)
    x[1, :128] = 1e-38                                                 # below the floor of the scale
    x[2, 5] = 3e38
    x[3, 7] = float("inf")
    x[4, 9] = float("nan")
    x[5, 3], x[5, 4] = -448.0, 447.0
    codes, scales = (t.float().cpu() for t in B.dit_quantize_block128(x.cuda()))
    want_codes, want_scales = plain_quantize(x[[0, 1, 2, 5]], False)
    assert torch.equal(codes[[0, 1, 2, 5]], want_codes) and torch.equal(scales[:, [0, 1, 2, 5]], want_scales)
    assert scales[0, 3] == float("inf") and bool(codes[3, 7].isnan()) and scales[0, 4].isnan() and bool(codes[4, :128].isnan().all())
    assert not bool(codes[[3, 4], 128:].isnan().any())                 # the neighbouring group is untouched
    # a product with such a row is NaN in that row only
    b, bs = B.dit_quantize_weight_block128(torch.randn(256, 40, device="cuda"))
    a, sa = B.dit_quantize_block128(x.cuda())
    out = B.dit_gemm_block128(a, sa, b, bs, out_dtype=torch.float32).cpu()
    assert bool(out[[3, 4]].isnan().all()) and bool(out[[0, 1, 5]].isfinite().all())
    # row 2 is 3e38 * b[5]: beyond fp32's 3.4e38 wherever |b[5]| > 1.14, an infinity there, and nowhere a NaN
    assert not bool(out[2].isnan().any())


def operands(seed, m, n, k, pitch=None):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    pitch = pitch or (k + 15) // 16 * 16
    normal = lambda *s: torch.randn(*s, generator=g, device="cuda")
    code = lambda rows: (normal(rows, pitch) * 100).clamp(-448, 448).to(torch.float8_e4m3fn)[:, :k]
    groups = (k + 127) // 128
    return (code(m), torch.exp(normal(groups, m)) / 100, code(n), torch.exp(normal((n + 127) // 128, groups)) / 100, normal(n))


def definition(a, sa, b, sb, bias):
    """The product and the sum of its terms' magnitudes, in 64 bits."""
    import torch
    out, mag = 0.0, 0.0
    for g in range(sa.shape[0]):
        at = slice(128 * g, min(a.shape[1], 128 * g + 128))
        f = sa[g].double()[:, None] * sb[:, g].double().repeat_interleave(128)[:b.shape[0]][None]
        x, y = a[:, at].double(), b[:, at].double()
        out, mag = out + f * (x @ y.t()), mag + f * (x.abs() @ y.abs().t())
    return (out, mag) if bias is None else (out + bias.double(), mag + bias.double().abs())


def allowed(want, mag, groups, dtype):
    import torch
    t = (128 * 2.0 ** -23 + (groups + 3 + 8) * 2.0 ** -24) * mag
    if dtype == torch.float32:
        return t
    smallest = 2.0 ** -25 if dtype == torch.float16 else 0.0
    return t + torch.finfo(dtype).eps / 2 * (want.abs() + t) + smallest


def check(got, args, dtype):
    import torch
    want, mag = definition(*args)
    off = (got.double() - want).abs()
    room = allowed(want, mag, args[1].shape[0], dtype)
    assert got.dtype == dtype and bool((off <= room).all()), f"off by {float((off / room).max()):.2f} of what is allowed"


# rows around every tile width of the split kernel, columns and k off the blocks, and shapes of the pair kernel
@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (1, 128, 128), (1, 1000, 2056), (2, 129, 16), (16, 300, 127), (17, 64, 129), (32, 257, 384),
                                   (33, 130, 1160), (64, 100, 4096), (65, 513, 640), (128, 300, 260), (129, 1000, 700), (300, 255, 1111),
                                   (700, 640, 12288), (1536, 2304, 384), (2600, 1800, 300), (3000, 2050, 1000)])
@pytest.mark.parametrize("kind", ["float16", "bfloat16", "float32"])
def test_product_against_the_definition(B, m, n, k, kind):
    import torch
    args = operands(m + n + k, m, n, k)
    dtype = getattr(torch, kind)
    check(B.dit_gemm_block128(*args, out_dtype=dtype), args, dtype)
    if m in (1, 129, 2600):
        args = args[:4] + (None,)
        check(B.dit_gemm_block128(*args, out_dtype=dtype), args, dtype)
    B.dit_ops_poll_status()


@pytest.mark.parametrize("m,n", [(5, 200), (90, 333), (2400, 1700)])
@pytest.mark.parametrize("kind", ["float16", "float32"])
def test_product_ignores_the_pitch_and_writes_inside_its_rows_only(B, m, n, kind):
    """Codes past k are NaN, scale rows have a stride, the output starts off every boundary and has columns and rows of
    somebody else around it."""
    import torch
    k, dtype = 200, getattr(torch, kind)
    a, sa, b, sb, bias = operands(7, m, n, k, pitch=256)
    for t in (a, b):
        torch.as_strided(t.view(torch.uint8), (t.shape[0], 256), (256, 1))[:, k:] = 0x7F
    wide_sa = torch.full((2, m + 5), float("nan"), device="cuda")
    wide_sa[:, :m] = sa
    buf = torch.full((m + 2, n + 9), -3.0, dtype=dtype, device="cuda")
    out = buf[1:m + 1, 3:n + 3]
    B.dit_gemm_block128(a, wide_sa[:, :m], b, sb, bias, out=out)
    check(out, (a, sa, b, sb, bias), dtype)
    left = buf.clone()
    left[1:m + 1, 3:n + 3] = -3.0
    assert bool((left == -3.0).all())


def test_product_clamps_sixteen_bit_outputs(B):
    import torch
    a, sa, b, sb, _ = operands(9, 4, 130, 256)
    sa = sa * 1e9
    out = B.dit_gemm_block128(a, sa, b, sb, out_dtype=torch.float16)
    want, _ = definition(a, sa, b, sb, None)
    assert bool((want.abs() > 1e5).any()) and bool(out.isfinite().all()) and float(out.abs().max()) == 65504.0


@pytest.mark.parametrize("m,n,k", [(1, 1024, 1024), (100, 500, 2000), (2560, 2048, 512)])
def test_product_repeats_itself_on_other_streams_and_in_graphs(B, m, n, k):
    import torch
    args = operands(11, m, n, k)
    first = B.dit_gemm_block128(*args)
    x = draw(5, m, k, torch.float16).cuda()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = B.dit_gemm_block128(*args)
    third = B.dit_gemm_block128(*args, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(first, second) and torch.equal(first, third)
    graph, out = torch.cuda.CUDAGraph(), torch.empty_like(first)
    with torch.cuda.graph(graph):
        c2, s2 = B.dit_quantize_block128(x)
        B.dit_gemm_block128(c2, s2, args[2], args[3], out=out)
    x.mul_(0.5)                                                        # the replay reads what lies there now
    graph.replay()
    codes, scales = B.dit_quantize_block128(x)
    torch.cuda.synchronize()
    assert torch.equal(c2.float(), codes.float()) and torch.equal(s2, scales)
    check(out, (c2, s2, args[2], args[3], None), out.dtype)


def test_quantize_then_multiply_comes_near_the_unquantised_product(B):
    """Both operands' codes are off by at most half a step, 2^-4 of a value (or of the group's smallest normal code's
    step, 2^-10 of 2^-6 / 448 of its top), so a product is off by at most 2 * 2^-4 + 2^-8 of the sum of magnitudes plus
    the share of the subnormal codes."""
    import torch
    x, w = draw(1, 200, 700, torch.bfloat16, 0.3).cuda(), (draw(2, 700, 300, torch.bfloat16, 0.0) * 0.02).cuda()
    out = B.dit_gemm_block128(*B.dit_quantize_block128(x), *B.dit_quantize_weight_block128(w), out_dtype=torch.float32)
    want = x.double() @ w.double()
    mag = x.double().abs() @ w.double().abs()
    off = (out.double() - want).abs()
    assert bool((off <= (2 * 2.0 ** -4 + 2.0 ** -8) * mag + 2.0 ** -9).all())
    # rounding errors are independent: in the 2-norm the product is far nearer than the bound
    assert float(off.norm() / want.norm()) <= 2.0 ** -4

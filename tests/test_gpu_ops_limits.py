"""The context-free operators at the edges of what their headers allow: element offsets beyond 32 bits, calls that run at the same
time on two streams, tensors of a device that is not current, and waits that have not run out."""
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


@pytest.mark.parametrize("q_rows", [1, 130])
def test_attention_and_selection_beyond_32_bit_offsets(B, q_rows):
    """800 000 keys of 24 heads of 128: 2.4e9 elements each of k and v; everything is zero but two blocks at the far end."""
    import torch
    heads, dim, kv = 24, 128, 800_000
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.zeros(kv, heads * dim, dtype=torch.float16, device="cuda") for _ in range(2))
    q = torch.randn(q_rows, heads * dim, generator=g, device="cuda").half()
    last = kv // 128 - 1                                               # 800000 = 6250 * 128
    for j in (last, last - 7):
        k[128 * j:128 * j + 128] = torch.randn(128, heads * dim, generator=g, device="cuda").half() + q[:128].mean(0)
        v[128 * j:128 * j + 128] = torch.randn(128, heads * dim, generator=g, device="cuda").half()
    index, count = B.dit_select_blocks(q, k, [q_rows], [kv], heads, [2])
    assert index[:, 0].tolist() == [[last - 7, last]] * heads and bool((count == 2).all())
    out = B.dit_block_attention(q, k, v, [q_rows], [kv], heads, index, count)
    B.dit_ops_poll_status()
    n_first = min(q_rows, 128)
    keys = torch.cat([torch.arange(128 * j, 128 * j + 128, device="cuda") for j in (last - 7, last)])
    s = torch.einsum("qhd,khd->hqk", q[:n_first].double().view(-1, heads, dim), k[keys].double().view(-1, heads, dim)) * dim ** -0.5
    want = torch.einsum("hqk,khd->qhd", torch.softmax(s, 2), v[keys].double().view(-1, heads, dim)).reshape(n_first, -1)
    # probabilities and results rounded to fp16, 256 keys with values of up to six: see the bounds of the attention's own tests
    assert float((out[:n_first].double() - want).abs().max()) <= (2 * 2.0 ** -11 + 2.0 ** -14) * float(v[keys].abs().max())
    assert bool(out.isfinite().all())


def test_product_and_quantiser_beyond_32_bit_offsets(B):
    """A [66000, 33000] output and input: 2.2e9 elements; the rows at the far end are checked."""
    import torch
    m, n, k = 66_000, 33_000, 64
    g = torch.Generator(device="cuda").manual_seed(2)
    a, sa = B.dit_quantize_block128(torch.randn(m, k, generator=g, device="cuda"))
    b, sb = B.dit_quantize_weight_block128(torch.randn(k, n, generator=g, device="cuda"))
    out = B.dit_gemm_block128(a, sa, b, sb)
    B.dit_ops_poll_status()
    rows = torch.tensor([0, 40_000, m - 200, m - 1], device="cuda")
    want = (a[rows].double() * sa[0, rows].double()[:, None]) @ (b.double() * sb[:, 0].double().repeat_interleave(128)[:n, None]).t()
    # one group: fp32 sums of 64 products, two scalings and the rounding to fp16
    mag = (a[rows].double().abs() * sa[0, rows].double()[:, None]) @ (b.double().abs() * sb[:, 0].double().repeat_interleave(128)[:n, None]).t()
    assert bool(((out[rows].double() - want).abs() <= (70 * 2.0 ** -23) * mag + 2.0 ** -11 * want.abs() + 2.0 ** -25).all())
    codes, scales = B.dit_quantize_block128(out)
    tail_codes, tail_scales = B.dit_quantize_block128(out[-300:].clone())
    assert torch.equal(codes[-300:].float(), tail_codes.float()) and torch.equal(scales[:, -300:], tail_scales)


def test_operators_at_the_same_time_on_two_streams(B):
    """Kernels that take tensor memory, with and without clusters, next to each other: each result as when alone."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(3)
    heads, dim, L = 6, 64, [700, 1300, 90]
    q, k, v = (torch.randn(sum(L), heads * dim, generator=g, device="cuda").half() for _ in range(3))
    new = torch.randn(3, heads * dim, generator=g, device="cuda").half()
    index, count = B.dit_select_blocks(q, k, L, L, heads, [3, 4, 1])
    first = torch.zeros((heads, 3, 4), dtype=torch.int32, device="cuda")
    ones = torch.ones((heads, 3), dtype=torch.int32, device="cuda")
    small = (*B.dit_quantize_block128(torch.randn(40, 2000, generator=g, device="cuda")), *B.dit_quantize_weight_block128(torch.randn(2000, 1500, generator=g, device="cuda")))
    large = (*B.dit_quantize_block128(torch.randn(2000, 512, generator=g, device="cuda")), *B.dit_quantize_weight_block128(torch.randn(512, 2048, generator=g, device="cuda")))
    calls = [lambda: B.dit_block_attention(q, k, v, L, L, heads, index, count), lambda: B.dit_gemm_block128(*small), lambda: B.dit_gemm_block128(*large),
             lambda: B.dit_block_attention(new, k, v, [1, 1, 1], L, heads, first, ones), lambda: B.dit_select_blocks(q, k, L, L, heads, [3, 4, 1])[0]]
    want = [c() for c in calls]
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    got = []
    for i in range(60):
        with torch.cuda.stream(streams[i % 3]):
            got.append((i, calls[(i * 7 + i // 5) % len(calls)]()))
    torch.cuda.synchronize()
    B.dit_ops_poll_status()
    for i, out in got:
        assert torch.equal(out, want[(i * 7 + i // 5) % len(calls)]), i


def test_a_tensor_on_another_device_is_refused_or_served_there(B):
    import torch
    x = torch.randn(4, 256, device="cuda")
    with pytest.raises(B.DitError):
        B.dit_quantize_block128(x, scales=torch.empty(2, 4))           # host memory
    if torch.cuda.device_count() > 1:                                  # the call makes the tensors' device current
        y = torch.randn(4, 256, device="cuda:1")
        codes, scales = B.dit_quantize_block128(y)
        assert codes.device == y.device and torch.cuda.current_device() == 0
        with pytest.raises(B.DitError):
            B.dit_quantize_block128(y, stream=torch.cuda.Stream(device="cuda:0"))
        with pytest.raises(B.DitError):
            B.dit_quantize_block128(y, scales=torch.empty(2, 4, device="cuda:0"))


def test_binding_refuses_mismatched_arguments(B):
    import torch
    q = torch.zeros(10, 128, dtype=torch.float16, device="cuda")
    index, count = torch.zeros(2, 1, 1, dtype=torch.int32, device="cuda"), torch.ones(2, 1, dtype=torch.int32, device="cuda")
    good = dict(q=q, k=q, v=q, q_lens=[10], kv_lens=[10], n_heads=2, index=index, count=count)
    B.dit_block_attention(**good)
    for kw in (dict(q_lens=[9]), dict(kv_lens=[11]), dict(kv_lens=[5, 5]), dict(k=q.bfloat16()), dict(v=q[:5]), dict(n_heads=3), dict(index=index.long()),
               dict(index=index[:, :, :0].expand(2, 2, 0)), dict(count=count[:1]), dict(q=q.float()), dict(q=q.t()), dict(scale=-0.1), dict(out=q[:5]), dict(v=None),
               dict(k=torch.zeros(10, 256, dtype=torch.float16, device="cuda")[:, ::2])):
        with pytest.raises(B.DitError):
            B.dit_block_attention(**{**good, **kw})
    for kw in (dict(keep=[0]), dict(keep=[1, 1]), dict(keep=[1], tail_rows=[-1]), dict(keep=[1], tail_rows=[]), dict(keep=[2], index=index)):
        with pytest.raises(B.DitError):
            B.dit_select_blocks(q, q, [10], [10], 2, **kw)
    a, sa = B.dit_quantize_block128(q)
    for kw in (dict(b=a[:, :64]), dict(a_scales=sa.t()), dict(b_scales=sa), dict(bias=torch.zeros(9, device="cuda")), dict(bias=torch.zeros(10, device="cuda").half()),
               dict(out=torch.zeros(10, 9, device="cuda")), dict(a=q), dict(out_dtype=torch.int32), dict(out=torch.zeros(10, 10, device="cuda"), out_dtype=torch.float16)):
        with pytest.raises(B.DitError):
            B.dit_gemm_block128(**{**dict(a=a, a_scales=sa, b=a, b_scales=sa[:, :1].contiguous()), **kw})
    with pytest.raises(B.DitError):
        B.dit_quantize_block128(q[0])
    with pytest.raises(B.DitError):
        B.dit_quantize_block128(q.int())


@pytest.mark.parametrize("rows", [1, 4])
def test_scales_whose_groups_share_their_memory_are_refused(B, rows):
    """An expanded [1, rows] matrix has room for one group; it has the shape of all of them."""
    import torch
    x = torch.ones(rows, 512, device="cuda")
    codes, scales = B.dit_quantize_block128(x)
    w, sw = B.dit_quantize_weight_block128(torch.ones(512, 128, device="cuda"))
    shared = torch.full((1, 1), -1.0, device="cuda").expand(4, rows) if rows == 1 else torch.full((1, rows), -1.0, device="cuda").expand(4, rows)
    with pytest.raises(B.DitError):
        B.dit_quantize_block128(x, scales=shared)
    with pytest.raises(B.DitError):
        B.dit_gemm_block128(codes, shared, w, sw)
    assert bool((shared == -1.0).all())
    apart = torch.full((4, rows + 3), -1.0, device="cuda")             # a wider matrix is served, its rest left alone
    B.dit_quantize_block128(x, scales=apart[:, :rows])
    assert torch.equal(apart[:, :rows], scales) and bool((apart[:, rows:] == -1.0).all())
    assert torch.equal(B.dit_gemm_block128(codes, apart[:, :rows], w, sw), B.dit_gemm_block128(codes, scales, w, sw))


def test_what_a_call_allocates_belongs_to_the_stream_it_is_given(B):
    """Results and the selector's workspace; from the current stream's memory they could be handed out again, or still be in use, while
    the kernels run on the other stream."""
    import torch
    heads, dim, L = 4, 128, [128 * 2000]
    q = torch.randn(L[0], heads * dim, device="cuda").half()
    w, sw = B.dit_quantize_weight_block128(torch.randn(heads * dim, 512, device="cuda"))
    want = [B.dit_quantize_block128(q), B.dit_select_blocks(q, q, L, L, heads, [3])]
    want += [(B.dit_gemm_block128(*want[0], w, sw),), (B.dit_block_attention(q, q, q, L, L, heads, *want[1]),)]
    side = torch.cuda.Stream()

    def owner(address):
        for s in torch.cuda.memory_snapshot():
            if s["address"] <= address < s["address"] + s["total_size"]:
                return s["stream"]

    def held():
        return sum(s["total_size"] for s in torch.cuda.memory_snapshot() if s["stream"] == side.cuda_stream)
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    before = held()
    got = [B.dit_select_blocks(q, q, L, L, heads, [3], stream=side)]
    assert held() - before >= 2 * 2000 * heads * dim * 8               # the workspace (16 MB): means of the blocks of q and k
    got = [B.dit_quantize_block128(q, stream=side)] + got
    got += [(B.dit_gemm_block128(*got[0], w, sw, stream=side),), (B.dit_block_attention(q, q, q, L, L, heads, *got[1], stream=side),)]
    torch.cuda.synchronize()
    for made, expected in zip(got, want):
        for x, y in zip(made, expected):
            assert owner(x.data_ptr()) == side.cuda_stream
            assert torch.equal(x.view(torch.uint8) if x.element_size() == 1 else x, y.view(torch.uint8) if y.element_size() == 1 else y)
    assert torch.cuda.current_stream() != side and torch.cuda.current_device() == 0


def test_lengths_that_change_while_they_are_read(B):
    import torch
    q = torch.zeros(10, 128, dtype=torch.float16, device="cuda")

    class Shrinking:
        def __index__(self):
            del lens[1:]
            return 4
    lens = [Shrinking()] + [3, 3]
    index, count = B.dit_select_blocks(q, q, lens, (4, 3, 3), 2, [1, 1, 1])
    assert len(lens) == 1 and index.shape == (2, 3, 1) and bool((count == 1).all())


def test_a_selector_asked_for_more_blocks_than_any_request_has(B):
    """keep = 2^31 - 1, as a caller may write `all of them`: every block, then -1 to the end of the list, and nothing around it.  (A 32-bit
    counter of the entries behind the last block would pass the largest int in its last step and go on in front of the list.)"""
    import torch
    if torch.cuda.mem_get_info()[0] < 20 << 30:
        pytest.skip("needs a list of 8.6 GB")
    keep, pad = 2 ** 31 - 1, 4096
    q = torch.randn(300, 64, device="cuda").half()
    buf = torch.full((keep + 2 * pad,), 7, dtype=torch.int32, device="cuda")
    index = buf[pad:pad + keep].view(1, 1, keep)
    count = torch.empty(1, 1, dtype=torch.int32, device="cuda")
    B.dit_select_blocks(q[:100], q, [100], [300], 1, [keep], index=index, count=count)
    torch.cuda.synchronize()
    assert count.tolist() == [[3]] and index[0, 0, :3].tolist() == [0, 1, 2]
    assert bool((buf[:pad] == 7).all()) and bool((buf[pad + keep:] == 7).all())
    assert int(buf[pad + 3:pad + keep].max()) == -1 and int(buf[pad + 3:pad + keep].min()) == -1


def test_a_scale_that_fp32_cannot_tell_from_zero_is_refused(B):
    """Zero stands for 1 / sqrt(head_dim): a tiny or negative number that rounds to it must not be taken for that."""
    import torch
    q = torch.randn(10, 128, dtype=torch.float16, device="cuda")
    index, count = torch.zeros(2, 1, 1, dtype=torch.int32, device="cuda"), torch.ones(2, 1, dtype=torch.int32, device="cuda")
    call = lambda scale: B.dit_block_attention(q, q, q, [10], [10], 2, index, count, scale=scale)
    for scale in (1e-46, 5e-324, -1e-46, -1e-300):
        with pytest.raises(B.DitError) as e:
            call(scale)
        assert e.value.status == 1
    assert torch.equal(call(0.0), call(-0.0)) and torch.equal(call(0.0), call(64 ** -0.5))
    # the smallest number that fp32 has: every key counts alike
    assert float((call(1e-45).double() - q.double().mean(0)).abs().max()) <= 2.0 ** -10 * float(q.abs().max())

"""A prompt encoder's layer in reduced arithmetic out of the context-free operators, as a caller would run it, and the operators at the edges of what
their headers allow."""
import ctypes as C

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


class Layer:
    """norm-free attention layer: x + out(attention(rotary(qkv(x)))), both products in 4 bits.  It keeps its weights' codes."""

    def __init__(self, B, hidden, heads, kv_heads, dim, group, seed):
        import torch
        g = torch.Generator().manual_seed(seed)
        self.B, self.heads, self.kv_heads, self.dim, self.group, self.hidden = B, heads, kv_heads, dim, group, hidden
        width = (heads + 2 * kv_heads) * dim
        self.w_qkv = (torch.randn(hidden, width, generator=g) * hidden ** -0.5).bfloat16().cuda()
        self.w_out = (torch.randn(heads * dim, hidden, generator=g) * (heads * dim) ** -0.5).bfloat16().cuda()
        self.b_qkv = (0.1 * torch.randn(width, generator=g)).cuda()
        self.qkv_codes, self.out_codes = B.dit_quantize_weight_fp4(self.w_qkv, group), B.dit_quantize_weight_fp4(self.w_out, group)

    def product(self, x, weight, k, bias, dtype):
        a = self.B.dit_quantize_fp4(x, self.group)
        return self.B.dit_gemm_fp4(a[0], a[1], weight[0], weight[1], k, self.group, a[2], weight[2], bias=bias, out_dtype=dtype)

    def __call__(self, x, lens, first, cache=None, kv_lens=None):
        """x [rows, hidden] fp16.  cache: (k, v) of whole contexts whose last rows are x's, written before."""
        h, g, d = self.heads, self.kv_heads, self.dim
        qkv = self.product(x, self.qkv_codes, self.hidden, self.b_qkv, x.dtype)
        turned = qkv[:, :(h + g) * d]
        self.B.dit_rotary(turned, h + g, lens, first=first, base=500000.0, factor=4.0, ramp=(1, 4, 512), out=turned)
        q, k, v = qkv[:, :h * d], qkv[:, h * d:(h + g) * d], qkv[:, (h + g) * d:]
        if cache is not None:
            for t, new in zip(cache, (k, v)):
                t[np.cumsum(kv_lens) - 1] = new                          # single rows: the last of each context
            k, v = cache
        mixed = self.B.dit_prompt_attention(q, k, v, lens, kv_lens or lens, h, g)
        return x + self.product(mixed, self.out_codes, h * d, None, x.dtype), (qkv, mixed)


def f64(t):
    return t.double().cpu().numpy()


def linear(a, w, group, bias=0.0):
    """(a w with both operands quantised, how far sums of products in fp32 may be off), in 64 bits."""
    qa, qw = P.quantize(f64(a), group), P.quantize(f64(w).T, group)
    va, vw = P.values(*qa, group), P.values(*qw, group)
    return va @ vw.T + bias, (np.abs(va) @ np.abs(vw).T) * (a.shape[1] + 12) * 2.0 ** -23


def check_output(y, x, mixed, w, group):
    """x + mixed w: the product rounded to fp16, then the sum."""
    want, off = linear(mixed, w, group)
    total = f64(x) + want
    assert (np.abs(f64(y) - total) <= (off + 2.0 ** -11 * np.abs(want) + 2.0 ** -25) * (1 + 2.0 ** -11) + 2.0 ** -11 * np.abs(total) + 2.0 ** -25).all()


@pytest.mark.parametrize("group", [16, 32])
def test_a_layer_stage_by_stage(B, group):
    """Each stage against the oracle's on the GPU's own input to it.  A product is off by k * 2^-23 of its magnitudes and half a step of fp16 (and of
    what it is added to); a rotation by 2^-21 of its pair and half a step; attention as counted in its own test, here rounded up."""
    import torch
    layer = Layer(B, 384, 6, 2, 64, group, 1)
    lens, first = [77, 5, 130], [0, 3, 1000]
    x = torch.randn(sum(lens), 384, generator=torch.Generator().manual_seed(2)).half().cuda()
    y, (qkv, mixed) = layer(x, lens, first)
    B.dit_ops_poll_status()
    want, off = linear(x, layer.w_qkv, group, f64(layer.b_qkv))
    turned = P.rotary(want[:, :8 * 64], np.concatenate([np.arange(f, f + l) for l, f in zip(lens, first)]), 8, P.frequencies(64, 500000.0, 4.0, (1, 4, 512)))
    got = f64(qkv)
    # rounded to fp16 before the rotation and after it, the first rounding and the product's error spread over the pair
    pair = np.abs(want[:, :512]).reshape(-1, 8, 2, 32)
    pair = np.broadcast_to(pair.sum(2, keepdims=True), pair.shape).reshape(-1, 512)
    both = off[:, :512].reshape(-1, 8, 2, 32)
    both = np.broadcast_to(both.sum(2, keepdims=True), both.shape).reshape(-1, 512)
    assert (np.abs(got[:, :512] - turned) <= both + pair * (2.0 ** -11 + 2.0 ** -20) + 2.0 ** -11 * np.abs(turned) + 2.0 ** -23).all()
    assert (np.abs(got[:, 512:] - want[:, 512:]) <= off[:, 512:] + 2.0 ** -11 * np.abs(want[:, 512:]) + 2.0 ** -24).all()
    att = P.attention(got[:, :384], got[:, 384:512], got[:, 512:], lens, lens, 6, 2)
    assert np.abs(f64(mixed) - att).max() <= 4 * 2.0 ** -11 * np.abs(got[:, 512:]).max()
    check_output(y, x, mixed, layer.w_out, group)


def test_a_new_row_at_a_time_gives_what_the_whole_prompt_gives(B):
    """The last row of three prompts through the layer alone, against the stored keys and values of the others.  Its codes are the same; its products are
    summed in another order (a step of fp16 at most), and so is its attention (a step each way, probabilities rounded on both sides); the product
    behind it is then checked against its own input, since four-bit codes turn a step of fp16 into one of theirs."""
    import torch
    layer = Layer(B, 384, 6, 2, 64, 16, 3)
    lens = [300, 41, 129]
    x = torch.randn(sum(lens), 384, generator=torch.Generator().manual_seed(4)).half().cuda()
    _, (qkv, mixed) = layer(x, lens, [0, 0, 0])
    last = np.cumsum(lens) - 1
    cache = [qkv[:, 384:512].clone(), qkv[:, 512:].clone()]
    for t in cache:
        t[last] = float("nan")                                           # to be written by the call
    one, (qkv1, mixed1) = layer(x[last], [1, 1, 1], [l - 1 for l in lens], cache, lens)
    # (a product of three rows is summed in another order than one of 470: rounded to fp16 they differ by a step at most)
    assert (qkv1 - qkv[last]).abs().max() <= 2.0 ** -10 * qkv[last].abs().max()
    assert (mixed1.double() - mixed[last].double()).abs().max() <= 8 * 2.0 ** -11 * qkv[:, 512:].abs().max()
    check_output(one, x[last], mixed1, layer.w_out, 16)


def test_a_captured_layer(B):
    import torch
    layer = Layer(B, 384, 6, 2, 64, 16, 5)
    lens = [40, 300, 1]
    x = torch.randn(sum(lens), 384, generator=torch.Generator().manual_seed(6)).half().cuda()
    x2 = torch.randn(sum(lens), 384, generator=torch.Generator().manual_seed(7)).half().cuda()
    want, want2 = layer(x, lens, [0, 0, 9])[0], layer(x2, lens, [0, 0, 9])[0]
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        got, _ = layer(x, lens, [0, 0, 9])
    for source, result in ((x2, want2), (x.clone(), want)):
        x.copy_(source)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, result)
    B.dit_ops_poll_status()


def test_operators_at_the_same_time_on_three_streams(B):
    """Kernels that take all of tensor memory, half of it or none, with and without clusters, next to each other: each result as when alone."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(3)
    n = lambda *s: torch.randn(*s, generator=g, device="cuda")
    small = (B.dit_quantize_fp4(n(40, 2000)), B.dit_quantize_weight_fp4(n(2000, 1500)))
    large = (B.dit_quantize_fp4(n(2000, 512), 32), B.dit_quantize_weight_fp4(n(512, 2048), 32))
    e4m3 = (*B.dit_quantize_block128(n(2000, 512)), *B.dit_quantize_weight_block128(n(512, 2048)))
    lens = [700, 1300, 90]
    q, k, v = n(sum(lens), 12 * 64).half(), n(sum(lens), 4 * 64).half(), n(sum(lens), 4 * 64).half()
    new = n(3, 12 * 64).half()
    x = n(500, 3000).half()
    product = lambda ab, k_, group: B.dit_gemm_fp4(ab[0][0], ab[0][1], ab[1][0], ab[1][1], k_, group, ab[0][2], ab[1][2])
    calls = [lambda: product(small, 2000, 16), lambda: product(large, 512, 32), lambda: B.dit_prompt_attention(q, k, v, lens, lens, 12, 4),
             lambda: B.dit_prompt_attention(new, k, v, [1, 1, 1], lens, 12, 4), lambda: B.dit_gemm_block128(*e4m3), lambda: B.dit_quantize_fp4(x)[0],
             lambda: B.dit_rotary(q, 12, lens)]
    want = [c() for c in calls]
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    got = []
    for i in range(84):
        with torch.cuda.stream(streams[i % 3]):
            got.append((i, calls[(i * 5 + i // 7) % len(calls)]()))
    torch.cuda.synchronize()
    B.dit_ops_poll_status()
    for i, out in got:
        assert torch.equal(out, want[(i * 5 + i // 7) % len(calls)]), i


def test_what_a_call_allocates_belongs_to_the_stream_it_is_given(B):
    import torch
    side = torch.cuda.Stream()
    x = torch.randn(300, 768, device="cuda").half()
    w = B.dit_quantize_weight_fp4(torch.randn(768, 512, device="cuda"))
    q = torch.randn(2, 8 * 128, device="cuda").half()
    k = torch.randn(20000, 128, device="cuda").half()

    def run(**kw):
        a = B.dit_quantize_fp4(x, **kw)
        return [*a, B.dit_dequantize_fp4(a[0], a[1], 768, 16, a[2], **kw), B.dit_gemm_fp4(a[0], a[1], w[0], w[1], 768, 16, a[2], w[2], **kw), B.dit_rotary(x, 6, [300], **kw),
                B.dit_prompt_attention(q, k, k, [1, 1], [9000, 11000], 8, 1, **kw)]
    want = run()

    def owner(address):
        for s in torch.cuda.memory_snapshot():
            if s["address"] <= address < s["address"] + s["total_size"]:
                return s["stream"]

    def held():
        return sum(s["active_size"] for s in torch.cuda.memory_snapshot() if s["stream"] == side.cuda_stream)
    torch.cuda.synchronize()
    got = run(stream=side)
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert owner(a.data_ptr()) == side.cuda_stream and torch.equal(a, b)
    assert held() > 0 and torch.cuda.current_stream() != side and torch.cuda.current_device() == 0


def test_offsets_beyond_32_bits(B):
    """A [66000, 33000] output and input (2.2e9 elements), and 4.4e9 turned channels; the rows at the far end are checked."""
    import torch
    m, n, k = 66_000, 33_000, 64
    g = torch.Generator(device="cuda").manual_seed(2)
    a = B.dit_quantize_fp4(torch.randn(m, k, generator=g, device="cuda"))
    b = B.dit_quantize_fp4(torch.randn(n, k, generator=g, device="cuda"))
    out = B.dit_gemm_fp4(a[0], a[1], b[0], b[1], k, 16, a[2], b[2])
    B.dit_ops_poll_status()
    rows = torch.tensor([0, 40_000, m - 200, m - 1], device="cuda")
    va = B.dit_dequantize_fp4(a[0], a[1], k, 16, a[2], out_dtype=torch.float32).double()[rows]
    vb = B.dit_dequantize_fp4(b[0], b[1], k, 16, b[2], out_dtype=torch.float32).double()
    want = va @ vb.t()
    assert bool(((out[rows].double() - want).abs() <= 80 * 2.0 ** -23 * (va.abs() @ vb.abs().t()) + 2.0 ** -11 * want.abs() + 2.0 ** -25).all())
    codes, scales, row_scales = B.dit_quantize_fp4(out)
    tail = B.dit_quantize_fp4(out[-300:].clone())
    assert torch.equal(codes[-300:], tail[0]) and torch.equal(row_scales[-300:], tail[2])
    back = B.dit_dequantize_fp4(codes, scales, n, 16, row_scales)
    assert torch.equal(back[-300:], B.dit_dequantize_fp4(tail[0], tail[1], n, 16, tail[2]))
    del back, codes, scales
    turned = B.dit_rotary(out, 250, [m], rotary_dim=132)                 # heads of 132, the pieces of 8 bytes
    assert torch.equal(turned[-300:], B.dit_rotary(out[-300:].clone(), 250, [300], first=[m - 300], rotary_dim=132))
    del turned
    w = B.dit_quantize_weight_fp4(out, 32)                               # [33000, 66000] codes
    assert torch.equal(w[0][-300:], B.dit_quantize_weight_fp4(out[:, -300:].contiguous(), 32)[0])


def test_binding_refuses_mismatched_arguments(B):
    import torch
    x = torch.zeros(10, 128, dtype=torch.float16, device="cuda")
    codes, scales, rows = B.dit_quantize_fp4(x)
    for kw in (dict(group=8), dict(codes=codes[:5]), dict(codes=codes.char()), dict(codes=codes[:, :32]), dict(scales=scales[:, :1]), dict(scales=scales.float()), dict(row_scales=rows[:9]),
               dict(row_scales=rows.half()), dict(group=32, row_scales=rows), dict(codes=torch.empty(10, 70, dtype=torch.uint8, device="cuda")[:, :64]), dict(codes=codes[:1].expand(10, 64)),
               dict(codes=codes.cpu()), dict(scales=scales.cpu())):
        with pytest.raises(B.DitError):
            B.dit_quantize_fp4(x, **kw)
    for bad in (x[0], x.int(), x[:, ::2], x.cpu(), x[:, :0]):
        with pytest.raises(B.DitError):
            B.dit_quantize_fp4(bad)
    good = dict(a=codes, a_scales=scales, b=codes, b_scales=scales, k=128, group=16, a_row_scales=rows, b_row_scales=rows)
    assert B.dit_gemm_fp4(**good).shape == (10, 10)
    for kw in (dict(k=126), dict(k=130), dict(k=0), dict(group=32), dict(b=codes[:, :32]), dict(a_scales=scales[:, :1]), dict(b_scales=scales[0]), dict(a_row_scales=rows[:3]),
               dict(bias=torch.zeros(9, device="cuda")), dict(bias=torch.zeros(10, device="cuda").half()), dict(out=torch.zeros(10, 9, device="cuda")), dict(a=x), dict(out_dtype=torch.int32),
               dict(out=torch.zeros(10, 10, device="cuda"), out_dtype=torch.float16), dict(out_dtype=3), dict(k="a"), dict(k=1.5)):
        with pytest.raises(B.DitError):
            B.dit_gemm_fp4(**{**good, **kw})
    for kw in (dict(cols=126), dict(group=32), dict(out=x.float(), out_dtype=torch.float16), dict(out=x[:5]), dict(row_scales=rows[:4]), dict(scales=scales[:, :1])):
        with pytest.raises(B.DitError):
            B.dit_dequantize_fp4(**{**dict(codes=codes, scales=scales, cols=128, group=16, row_scales=rows), **kw})
    places = torch.zeros(10, dtype=torch.int32, device="cuda")
    for kw in (dict(), dict(lens=[9]), dict(lens=[10], positions=places), dict(positions=places[:9]), dict(positions=places.long()), dict(positions=places.cpu()), dict(positions=places, first=[0]),
               dict(lens=[10], first=[0, 0]), dict(lens=[10], first=[-1]), dict(lens=[11, -1]), dict(lens=[10], rotary_dim=3), dict(lens=[10], rotary_dim=130), dict(lens=[10], rotary_dim=0),
               dict(lens=[10], factor=0.5), dict(lens=[10], base=-1.0), dict(lens=[10], ramp=(1, 2)), dict(lens=[10], ramp=(2, 1, 100)), dict(lens=[10], ramp=(1, 2, 0)), dict(lens=[10], ramp=7),
               dict(lens=[10], magnitude="x"), dict(lens=[10], out=x[:5]), dict(lens=[10], out=x.float()), dict(lens=[2 ** 31]), dict(lens=[10], x=x.t()), dict(lens=[10], n_heads=3),
               dict(lens=[10], magnitude=float("inf")), dict(lens=[10], x=x.int())):
        with pytest.raises(B.DitError):
            B.dit_rotary(**{**dict(x=x, n_heads=2), **kw})
    good = dict(q=x, k=x, v=x, q_lens=[10], kv_lens=[10], n_heads=2)
    B.dit_prompt_attention(**good)
    for kw in (dict(q_lens=[9]), dict(kv_lens=[11]), dict(kv_lens=[5, 5]), dict(k=x.bfloat16()), dict(v=x[:5]), dict(n_heads=3), dict(n_kv_heads=1), dict(n_kv_heads=0), dict(n_kv_heads=4),
               dict(q=x.float(), k=x.float(), v=x.float()), dict(q=x.t()), dict(scale=-0.1), dict(scale=1e-46), dict(out=x[:5]), dict(v=None), dict(n_heads=4), dict(out=x.float()),
               dict(workspace=torch.empty(4)), dict(q_lens=[-1, 11], kv_lens=[10, 0]), dict(q_lens=[0] * 65, kv_lens=[0] * 65)):
        with pytest.raises(B.DitError):
            B.dit_prompt_attention(**{**good, **kw})
    with pytest.raises(B.DitError):                                      # too small a workspace
        B.dit_prompt_attention(x[:1], x.expand(10, 128), x, [1], [10], 2, workspace=torch.empty(0, dtype=torch.uint8)) 
    if torch.cuda.device_count() > 1:                                    # the call makes the tensors' device current
        y = x.to("cuda:1")
        assert B.dit_rotary(y, 2, [10]).device == y.device and B.dit_quantize_fp4(y)[0].device == y.device and torch.cuda.current_device() == 0
        with pytest.raises(B.DitError):
            B.dit_quantize_fp4(y, codes=codes)


def test_inputs_that_require_a_gradient_are_taken_as_they_are(B):
    import torch
    x = torch.randn(5, 128, device="cuda", requires_grad=True)
    for out in (B.dit_quantize_fp4(x)[2], B.dit_rotary(x, 2, [5]), B.dit_prompt_attention(*(x.half(),) * 3, [5], [5], 2)):
        assert not out.requires_grad
    with pytest.raises(B.DitError):
        B.dit_rotary(torch._neg_view(x.detach()), 2, [5])                # lazily negated


@pytest.mark.parametrize("lens,contexts", [([1] * 9, [700] * 9), ([300, 1, 77], [300, 2000, 90]), ([900, 31], [900, 31])])
def test_calls_on_the_heels_of_one_another_wait_for_one_another(B, lens, contexts):
    """Operators set themselves up while the one in front of them ends.  A run of layers without a pause, whose intermediate tensors take one another's
    memory, gives bit for bit what the same calls give with a synchronisation behind each."""
    import torch
    layer = Layer(B, 384, 6, 2, 64, 16, 5)
    h, g, d, rows = 6, 2, 64, sum(lens)
    gen = torch.Generator().manual_seed(6)
    x = torch.randn(rows, 384, generator=gen).half().cuda()
    keys, values = (torch.randn(sum(contexts), g * d, generator=gen).half().cuda() for _ in range(2))
    first = [c - l for l, c in zip(lens, contexts)]
    mixed, out = (torch.empty(rows, 384, dtype=torch.float16, device="cuda") for _ in range(2))
    qkv = torch.empty(rows, (h + 2 * g) * d, dtype=torch.float16, device="cuda")

    def run(pause):
        results, y = [], x
        for i in range(12):
            a = B.dit_quantize_fp4(y, 16); pause()
            B.dit_gemm_fp4(a[0], a[1], layer.qkv_codes[0], layer.qkv_codes[1], 384, 16, a[2], layer.qkv_codes[2], bias=layer.b_qkv, out=qkv); pause()
            B.dit_rotary(qkv[:, :(h + g) * d], h + g, lens, first=first, out=qkv[:, :(h + g) * d]); pause()
            B.dit_rotary(keys, g, contexts, out=keys); pause()           # what attention reads has just been written
            B.dit_prompt_attention(qkv[:, :h * d], keys, values, lens, contexts, h, g, out=mixed); pause()
            a = B.dit_quantize_fp4(mixed, 16); pause()
            B.dit_gemm_fp4(a[0], a[1], layer.out_codes[0], layer.out_codes[1], h * d, 16, a[2], layer.out_codes[2], out=out); pause()
            back = B.dit_dequantize_fp4(a[0], a[1], h * d, 16, a[2], out_dtype=torch.float16); pause()
            B.dit_rotary(keys, g, contexts, inverse=True, out=keys); pause()
            y = out.clone() if i % 2 else out                            # (torch's kernels in between as well)
            results += [qkv.clone(), mixed.clone(), out.clone(), back]
        return results

    saved = keys.clone()
    want = run(torch.cuda.synchronize)
    keys.copy_(saved)
    got = run(lambda: None)
    graph, start = torch.cuda.CUDAGraph(), saved.clone()
    with torch.cuda.graph(graph):                                        # the host is not in between then
        keys.copy_(start)
        captured = run(lambda: None)
    for results in (got, captured):
        if results is captured:
            graph.replay()
        B.dit_ops_poll_status()
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(want, results)):
            assert torch.equal(a.view(torch.int16), b.view(torch.int16)), i


def test_calls_on_two_streams_captured_into_one_graph(B):
    """Fork and join: a product on one stream, a rotation and mixed attention on another, and a product of both results; replayed on new inputs."""
    import torch
    layer = Layer(B, 384, 6, 2, 64, 32, 7)
    lens, gen = [260, 1, 33], torch.Generator().manual_seed(8)
    rows = sum(lens)
    x, qkv = torch.empty(rows, 384, dtype=torch.float16, device="cuda"), torch.empty(rows, 640, dtype=torch.float16, device="cuda")

    def work(other):
        main = torch.cuda.current_stream()
        turned = torch.empty_like(qkv)
        mixed = torch.empty_like(x)
        if other is not None:
            other.wait_stream(main)
        with torch.cuda.stream(other or main):
            turned.copy_(qkv)
            B.dit_rotary(turned[:, :512], 8, lens, out=turned[:, :512])
            B.dit_prompt_attention(turned[:, :384], turned[:, 384:512], turned[:, 512:], lens, lens, 6, 2, out=mixed)
        y = layer.product(x, layer.out_codes, 384, None, torch.float16)
        if other is not None:
            main.wait_stream(other)
        return layer.product(mixed + y, layer.out_codes, 384, None, torch.float32), turned, mixed

    def fill():
        x.copy_(torch.randn(rows, 384, generator=gen).half())
        qkv.copy_(torch.randn(rows, 640, generator=gen).half())

    fill()
    work(None)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = work(torch.cuda.Stream())
    for _ in range(3):
        fill()
        want = [t.clone() for t in work(None)]
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(captured, want):
            assert torch.equal(a, b)
    B.dit_ops_poll_status()

"""Steps in reduced arithmetic: DIT_FLAG_FP8_BLOCK128 (block-scaled e4m3 products) and DIT_FLAG_SPARSE_ATTENTION (attention over
selected key blocks), alone and together.

Rounding to e4m3 and choosing blocks are discontinuous, so each stage is compared with the oracle's stage on the GPU's own
input to it (read through the taps): quantised codes are then the same on both sides, and what is left is
  * products: fp32 sums (128 * 2^-23 of the sum of magnitudes, a few 2^-24 more) and one rounding to fp16 (2^-11), GELU's tanh
    with the hardware's 2^-10.9 error of a value below 1: together below 2e-3 of a stage's rms for the maxima of 1e5 or more values
    of up to five rms each (fp16's 2^-11 * 5 rms = 2.4e-3 where a value is that large: hence 4e-3);
  * attention: probabilities and results rounded to fp16 (2 * 2^-11 of values of at most a few rms): below 4e-3 as well;
  * the block's output: fp32 throughout.  The 16-bit products add 16 terms at a time, each addition off by at most 2^-23 of the running
    sum (at most six rms of the branch over these 1e5 sums): K / 16 * 2^-23 * 6 of a branch's rms, 5.5e-4 for K = 12288 and 1.4e-4 for
    K = 3072: 7e-4 of the output's rms, which holds both gated branches (1e-4 was written here first, with the lengths left out).
The QKV product's own input does not survive the block (the second LayerNorm overwrites it), so q, k, v are compared with the oracle's
from the tokens on, where codes next to a rounding border may differ.  The GPU quantises h rounded to fp16: a value and the largest
of its group are each off by at most 2^-11, so a value over its scale by at most 2^-10; codes lie at least 2^-4 of their value apart, so
at most a share of 2^-10 / 2^-4 = 2^-6 of them falls on the other side of a border, each by a step of at most 2^-3 of its value:
an rms error of the operand of at most sqrt(2^-6) * 2^-3 = 1.56e-2, and of a product of independent terms as much (a first
bound of 3e-3 took no account of the group's largest value and of codes 2^-4 apart; typical errors of a third of the
largest give 4e-3).  A parallel block's h survives, and there q, k, v are held to the stage's bar as well."""
import numpy as np
import pytest

from oracle import block_oracle as K
from oracle import dit_oracle as O
from paper_2510_01565_b200 import workloads as W

pytestmark = pytest.mark.gpu

STAGE, OUTPUT, QKV_RMS = 4e-3, 7e-4, 1.6e-2


@pytest.fixture(scope="module")
def B():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("these tests need a CUDA device; the library has no CPU path")
    from paper_2510_01565_b200 import binding, build
    build.build_library()
    binding.load_library()
    return binding


def f64(w):
    return {k: W.bf16_to_f64(v) for k, v in w.items()}


def rms(x):
    return float(np.sqrt(np.mean(np.square(x))))


def keep_of(n_tokens, keep, least):
    n = -(-n_tokens // 128)
    return min(n, max(1, least, int(np.ceil(np.float64(np.float32(keep)) * n))))


def context(B, wl, flags, keep=None, least=1):
    slots = len(wl.weights)
    ctx = B.context_for(wl.dims, slots, wl.total_tokens, len(wl.requests), flags=flags)
    B.upload_weights(ctx, wl.weights)
    if keep is not None:
        ctx.dit_ctx_set_sparse_attention(keep, least)
    return ctx


def run(B, wl, ctx, with_geometry=True, requests=None):
    import torch
    which = list(range(len(wl.requests))) if requests is None else requests
    tok = B.bits_to_cuda_bf16(np.concatenate([wl.tokens[r] for r in which]))
    cond = B.bits_to_cuda_bf16(wl.cond[which])
    ctx.dit_debug_poison()
    if with_geometry:
        out = ctx.dit_step_forward_requests(tok, [wl.requests[r] for r in which], cond, len(wl.weights))
    else:
        out = ctx.dit_step_forward(tok, [wl.token_lens[r] for r in which], cond, len(wl.weights))
    torch.cuda.synchronize()
    ctx.dit_ctx_poll_status()
    B.dit_ops_poll_status()
    assert ctx.dit_debug_check_guards() == 0
    return out


@pytest.mark.parametrize("dims,reqs,keep", [(W.SMALL, [(384, 384, 77), (16, 16, 0), (160, 208, 9)], 0.4), (W.LARGE, [(512, 272, 130), (128, 96, 0)], 0.3)])
@pytest.mark.parametrize("quantised,sparse", [(True, False), (False, True), (True, True)])
def test_a_block_stage_by_stage(B, dims, reqs, keep, quantised, sparse):
    wl = W.make_custom("reduced", dims, 1, reqs, seed=51)
    w = f64(wl.weights[0])
    flags = (B.DIT_FLAG_FP8_BLOCK128 if quantised else 0) | (B.DIT_FLAG_SPARSE_ATTENTION if sparse else 0)
    ctx = context(B, wl, flags, keep if sparse else None)
    out = run(B, wl, ctx).double().cpu().numpy()
    taps = {n: ctx.dit_debug_tap(n).double().cpu().numpy() for n in ("h", "qkv", "attn", "u", "mod")}
    assert ctx.dit_last_launch_count() == 1 + 7 + (4 if quantised else 0) + (2 if sparse else 0)
    ctx.close()
    H, lin = dims.hidden, K.block_linear if quantised else (lambda a, ww, bb: a @ ww + bb)
    p = 0
    for r, n in enumerate(wl.token_lens):
        rows = slice(p, p + n)
        p += n
        x = W.bf16_to_f64(wl.tokens[r])
        shift_a, scale_a, gate_a, _, _, gate_m = O.adaln_modulation(W.bf16_to_f64(wl.cond[r]), w["w_ada"], w["b_ada"])
        qkv = lin(O.modulate(O.layer_norm(x, dims.ln_eps), shift_a, scale_a), w["w_qkv"], w["b_qkv"])
        assert rms(taps["qkv"][rows] - qkv) <= QKV_RMS * rms(qkv)
        q, k, v = (taps["qkv"][rows, i * H:(i + 1) * H] for i in range(3))
        if sparse:
            a = K.sparse_attention(q, k, v, dims.n_heads, K.select_blocks(q, k, dims.n_heads, keep_of(n, keep, 1), wl.requests[r].n_text_tokens))
        else:
            a = O.attention(q, k, v, dims.n_heads)
        assert np.abs(taps["attn"][rows] - a).max() <= STAGE * rms(a)
        u = O.gelu_tanh(lin(taps["h"][rows], w["w_fc1"], w["b_fc1"]))
        assert np.abs(taps["u"][rows] - u).max() <= STAGE * rms(u)
        y = x + gate_a * lin(taps["attn"][rows], w["w_o"], w["b_o"])
        y = y + gate_m * lin(taps["u"][rows], w["w_fc2"], w["b_fc2"])
        assert np.abs(out[rows] - y).max() <= OUTPUT * rms(y)


def test_stacks_of_both_forms_against_the_reduced_and_the_exact_block(B):
    """Two blocks, sequential and parallel, both reductions on: near the oracle's reduced stack (two quantised computations of the same
    numbers drift apart with depth, as in the e4m3 mode with row scales: 8e-2 there and here) and the exact dense one where nothing is left out."""
    wl = W.make_custom("reduced2", W.SMALL, 2, [(384, 384, 77), (160, 208, 9)], seed=52)
    wl.weights = [wl.weights[0], W.draw_parallel_block_weights(np.random.default_rng(52), wl.dims)]
    blocks = [f64(w) for w in wl.weights]
    both = B.DIT_FLAG_FP8_BLOCK128 | B.DIT_FLAG_SPARSE_ATTENTION
    ctx = context(B, wl, both, 0.5, 2)
    out = run(B, wl, ctx).double().cpu().numpy()
    assert ctx.dit_last_launch_count() == 1 + 7 + 5 + 4 + 2 + 2 * 2
    ctx.dit_ctx_set_sparse_attention(1.0)
    full = run(B, wl, ctx).double().cpu().numpy()
    ctx.close()
    p = 0
    for r, n in enumerate(wl.token_lens):
        x = y = z = W.bf16_to_f64(wl.tokens[r])
        for w in blocks:
            y = K.block_forward(y, W.bf16_to_f64(wl.cond[r]), w, wl.dims.n_heads, wl.dims.ln_eps, True, keep_of(n, 0.5, 2), wl.requests[r].n_text_tokens)
            z = O.any_block_forward(z, W.bf16_to_f64(wl.cond[r]), w, wl.dims.n_heads, wl.dims.ln_eps)
        assert rms(out[p:p + n] - y) <= 8e-2 * rms(y)
        assert rms(full[p:p + n] - z) <= 1e-1 * rms(z)
        p += n


@pytest.mark.parametrize("dims", [W.SMALL, W.LARGE])
def test_a_parallel_blocks_products(B, dims):
    wl = W.make_custom("reducedp", dims, 1, [(272, 256, 30), (64, 64, 1)], seed=59)
    wl.weights = [W.draw_parallel_block_weights(np.random.default_rng(59), dims)]
    w = f64(wl.weights[0])
    ctx = context(B, wl, B.DIT_FLAG_FP8_BLOCK128)
    out = run(B, wl, ctx).double().cpu().numpy()
    h, qkv = (ctx.dit_debug_tap(n).double().cpu().numpy() for n in ("h", "qkv"))
    ctx.close()
    want = K.block_linear(h, w["w_qkv"], w["b_qkv"])
    assert np.abs(qkv - want).max() <= STAGE * rms(want)
    u = O.gelu_tanh(K.block_linear(h, w["w_fc1"], w["b_fc1"]))
    p, H = 0, dims.hidden
    for r, n in enumerate(wl.token_lens):
        rows = slice(p, p + n)
        p += n
        gate = np.split(O.silu(W.bf16_to_f64(wl.cond[r])) @ w["w_ada"] + w["b_ada"], 3)[2]
        a = O.attention(qkv[rows, :H], qkv[rows, H:2 * H], qkv[rows, 2 * H:], dims.n_heads)
        x = W.bf16_to_f64(wl.tokens[r])
        branch = gate * K.block_linear(np.concatenate([a, u[rows]], axis=1), w["w_out"], w["b_out"])
        # [a | u] reaches the product rounded to fp16: the bound above for an operand, of the branch that it feeds
        assert rms(out[rows] - x - branch) <= QKV_RMS * rms(branch) + OUTPUT * rms(x)


@pytest.mark.parametrize("form", ["dual", "parallel_then_sequential", "qk_rope"])
def test_sparse_attention_in_the_other_block_forms(B, form):
    """The attention output of the last block against the oracle's selected attention on the GPU's own q, k, v, text rows kept."""
    reqs = [(384, 384, 77), (160, 208, 9), (64, 64, 200)]
    wl = W.make_custom("forms", W.SMALL, 2, reqs, seed=60)
    flags = B.DIT_FLAG_SPARSE_ATTENTION
    if form == "dual":
        wl.weights = [dict(wl.weights[0], txt=wl.weights[1])]
    elif form == "parallel_then_sequential":
        wl.weights = [W.draw_parallel_block_weights(np.random.default_rng(60), wl.dims), wl.weights[0]]
    else:
        flags |= B.DIT_FLAG_QK_RMSNORM | B.DIT_FLAG_ROPE_2D
    import torch
    ctx = B.context_for(wl.dims, 2, wl.total_tokens, 3, flags=flags)
    slots = B.upload_weights(ctx, wl.weights)
    ctx.dit_ctx_set_sparse_attention(0.45, 1)
    ctx.dit_debug_poison()
    out = ctx.dit_step_forward_requests(B.bits_to_cuda_bf16(wl.packed_tokens()), wl.requests, B.bits_to_cuda_bf16(wl.cond), slots)
    torch.cuda.synchronize()
    ctx.dit_ctx_poll_status()
    assert ctx.dit_debug_check_guards() == 0 and bool(out.isfinite().all())
    qkv, attn = (ctx.dit_debug_tap(n).double().cpu().numpy() for n in ("qkv", "attn"))
    ctx.close()
    p, H = 0, wl.dims.hidden
    for r, n in enumerate(wl.token_lens):
        rows = slice(p, p + n)
        p += n
        q, k, v = (qkv[rows, i * H:(i + 1) * H] for i in range(3))
        a = K.sparse_attention(q, k, v, wl.dims.n_heads, K.select_blocks(q, k, wl.dims.n_heads, keep_of(n, 0.45, 1), reqs[r][2]))
        assert np.abs(attn[rows] - a).max() <= STAGE * rms(a)


def test_keeping_everything_is_the_dense_step_bit_for_bit(B):
    import torch
    wl = W.make_custom("dense", W.SMALL, 2, [(256, 256, 3), (64, 64, 0)], seed=53)
    plain = context(B, wl, 0)
    want = run(B, wl, plain)
    plain.close()
    for flags in (B.DIT_FLAG_SPARSE_ATTENTION,):
        ctx = context(B, wl, flags)
        assert torch.equal(run(B, wl, ctx), want)                       # as created
        ctx.dit_ctx_set_sparse_attention(0.2, 3)                        # three blocks at least: both requests keep all of theirs
        assert torch.equal(run(B, wl, ctx, requests=[1]), want[-16:])
        ctx.dit_ctx_set_sparse_attention(1.0)
        assert torch.equal(run(B, wl, ctx), want)
        ctx.close()


@pytest.mark.parametrize("which", ["block128", "sparse", "both", "sparse_bf16", "sparse_qk", "sparse_e4m3"])
def test_host_steps_graphs_and_packing(B, which):
    """The host-buffer step and a replayed graph give the step's results; a request's lists do not depend on its neighbours, and where the
    products do not either (the 16-bit modes: tiles by position in the batch, one order of sums) neither does its output."""
    import torch
    flags = {"block128": B.DIT_FLAG_FP8_BLOCK128, "sparse": B.DIT_FLAG_SPARSE_ATTENTION, "both": B.DIT_FLAG_FP8_BLOCK128 | B.DIT_FLAG_SPARSE_ATTENTION,
             "sparse_bf16": B.DIT_FLAG_SPARSE_ATTENTION | B.DIT_FLAG_BF16_OPERANDS, "sparse_e4m3": B.DIT_FLAG_SPARSE_ATTENTION | B.DIT_FLAG_FP8_GEMM,
             "sparse_qk": B.DIT_FLAG_SPARSE_ATTENTION | B.DIT_FLAG_QK_RMSNORM | B.DIT_FLAG_ROPE_2D}[which]
    wl = W.make_custom("forms", W.SMALL, 2, [(384, 384, 77), (160, 208, 9), (512, 512, 0)], seed=54)
    sparse = bool(flags & B.DIT_FLAG_SPARSE_ATTENTION)
    ctx = context(B, wl, flags, 0.3 if sparse else None)
    want = run(B, wl, ctx)
    assert torch.equal(run(B, wl, ctx), want) and bool(want.isfinite().all())
    tok, cond = B.bits_to_cuda_bf16(wl.packed_tokens()), B.bits_to_cuda_bf16(wl.cond)
    geometry = lambda out: ctx.dit_step_forward_requests(tok, wl.requests, cond, 2, out=out)
    graph, replayed = torch.cuda.CUDAGraph(), torch.empty_like(want)
    with torch.cuda.graph(graph):
        geometry(replayed)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(replayed, want)
    if not flags & B.DIT_FLAG_ROPE_2D:
        lens_only = run(B, wl, ctx, with_geometry=False)                # without geometry no text rows are known
        host = torch.empty(want.shape, dtype=torch.float32).pin_memory()
        pin = lambda bits: torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).view(torch.bfloat16).pin_memory()
        ctx.dit_step_forward_host(pin(wl.packed_tokens()), wl.token_lens, pin(wl.cond), 2, host)
        assert torch.equal(host, lens_only.cpu())
    if not flags & B.DIT_FLAG_FP8_BLOCK128:
        assert torch.equal(run(B, wl, ctx, requests=[1]), want[wl.token_lens[0]:wl.token_lens[0] + wl.token_lens[1]])
    ctx.close()


def test_two_contexts_step_at_the_same_time(B):
    import torch
    both = B.DIT_FLAG_FP8_BLOCK128 | B.DIT_FLAG_SPARSE_ATTENTION
    wls = [W.make_custom(f"two{i}", W.SMALL, 2, [(384, 384, 7 + i), (160, 208, 9)], seed=55 + i) for i in range(2)]
    ctxs = [context(B, wl, both, 0.4) for wl in wls]
    want = [run(B, wl, ctx) for wl, ctx in zip(wls, ctxs)]
    ins = [(B.bits_to_cuda_bf16(wl.packed_tokens()), B.bits_to_cuda_bf16(wl.cond)) for wl in wls]
    outs, streams = [torch.empty_like(w) for w in want], [torch.cuda.Stream() for _ in wls]
    torch.cuda.synchronize()
    for _ in range(5):
        for i in range(2):
            ctxs[i].dit_step_forward_requests(ins[i][0], wls[i].requests, ins[i][1], 2, out=outs[i], stream=streams[i])
    torch.cuda.synchronize()
    for i in range(2):
        assert torch.equal(outs[i], want[i])
        ctxs[i].close()


def test_denoise_step_runs_reduced(B):
    import torch
    si = W.make_step_inputs(W.SMALL, 2, [(384, 384, 5), (32, 32, 0)], seed=57)
    ctx = B.context_for(si.dims, 2, sum(si.token_lens), 2, flags=B.DIT_FLAG_FP8_BLOCK128 | B.DIT_FLAG_SPARSE_ATTENTION)
    dense = B.context_for(si.dims, 2, sum(si.token_lens), 2)
    velocity = []
    for c in (ctx, dense):
        B.upload_weights(c, si.weights)
        B.upload_shell_weights(c, si.shell)
        if c is ctx:
            c.dit_ctx_set_sparse_attention(0.75)
        latents = torch.from_numpy(np.concatenate([z.reshape(-1) for z in si.latents])).cuda()
        v = torch.empty_like(latents)
        c.dit_denoise_step(latents, B.bits_to_cuda_bf16(np.concatenate(si.texts, axis=0)), si.requests, si.dsigmas, torch.from_numpy(si.pooled).cuda(), 2, velocity=v)
        torch.cuda.synchronize()
        c.dit_ctx_poll_status()
        velocity.append(v.double())
        c.close()
    off = float((velocity[0] - velocity[1]).norm() / velocity[1].norm())
    assert 1e-5 < off <= 2e-1                                           # a different computation, near the dense 16-bit one


def test_reduced_modes_refuse_what_they_were_not_built_for(B):
    wl = W.make_custom("refuse", W.SMALL, 2, [(64, 64, 3)], seed=58)
    for extra in (B.DIT_FLAG_QK_RMSNORM, B.DIT_FLAG_ROPE_2D, B.DIT_FLAG_FP8_GEMM, B.DIT_FLAG_BF16_OPERANDS):
        with pytest.raises(B.DitError) as e:
            B.context_for(wl.dims, 2, 64, 1, flags=B.DIT_FLAG_FP8_BLOCK128 | extra)
        assert e.value.status == 2
    ctx = B.context_for(wl.dims, 2, 64, 1, flags=B.DIT_FLAG_FP8_BLOCK128)
    dev = {k: B.bits_to_cuda_bf16(v) for k, v in wl.weights[0].items()}
    with pytest.raises(B.DitError) as e:
        ctx.dit_load_dual_block_weights(0, dev, dev)
    assert e.value.status == 2
    with pytest.raises(B.DitError) as e:
        ctx.dit_ctx_set_sparse_attention(0.5)
    assert e.value.status == 1
    ctx.close()
    ctx = B.context_for(wl.dims, 2, 64, 1, flags=B.DIT_FLAG_SPARSE_ATTENTION)
    for keep, least in ((0.0, 1), (-0.5, 1), (1.01, 1), (float("nan"), 1), (0.5, 0)):
        with pytest.raises(B.DitError) as e:
            ctx.dit_ctx_set_sparse_attention(keep, least)
        assert e.value.status == 1
    ctx.close()


def test_a_share_above_a_whole_number_of_blocks_takes_one_more(B):
    """ceil(keep * n), where only what rounding keep to fp32 adds (2^-24 of the product) is forgiven: 0.1 of ten blocks is one, the next
    float above 0.1 takes two, and the next above a half of two blocks takes both, which is the dense step bit for bit."""
    import torch
    above = lambda x: float(np.nextafter(np.float32(x), np.float32(1)))
    wl = W.make_custom("share", W.SMALL, 1, [(256, 256, 0), (512, 320, 640)], seed=61)
    assert wl.token_lens == [256, 1280]
    ctx = context(B, wl, B.DIT_FLAG_SPARSE_ATTENTION)

    def step(keep, least=1):
        ctx.dit_ctx_set_sparse_attention(keep, least)
        out = run(B, wl, ctx)
        return out[:256], out[256:]
    dense, one, two = step(1.0)[0], step(0.05)[1], step(0.15)[1]
    assert not torch.equal(step(0.5)[0], dense) and torch.equal(step(above(0.5))[0], dense)
    assert not torch.equal(one, two)
    assert torch.equal(step(0.1)[1], one) and torch.equal(step(above(0.1))[1], two) and torch.equal(step(0.2)[1], two)
    ctx.close()


def test_the_least_number_of_blocks_makes_a_short_request_dense(B):
    """Requests of three blocks and of one: with three blocks at least the step is the dense one bit for bit, with one at least it is not."""
    import torch
    wl = W.make_custom("least", W.SMALL, 2, [(256, 256, 3), (64, 64, 0)], seed=62)
    ctx = context(B, wl, B.DIT_FLAG_SPARSE_ATTENTION)
    want = run(B, wl, ctx)
    ctx.dit_ctx_set_sparse_attention(0.2, 3)
    assert torch.equal(run(B, wl, ctx), want)
    ctx.dit_ctx_set_sparse_attention(0.2, 1)
    assert not torch.equal(run(B, wl, ctx)[:259], want[:259])
    ctx.close()


@pytest.mark.parametrize("sparse", [False, True])
def test_host_steps_and_graphs_where_the_products_take_the_large_tiles(B, sparse):
    """4466 rows: the gated products run on 256 x 256 tiles, whose residual and output maps move with the host step's slices of rows; requests
    begin and end inside the slices and inside the tiles."""
    import torch
    flags = B.DIT_FLAG_FP8_BLOCK128 | (B.DIT_FLAG_SPARSE_ATTENTION if sparse else 0)
    wl = W.make_custom("slices", W.SMALL, 1, [(784, 784, 77), (160, 208, 9), (672, 704, 0), (16, 16, 0)], seed=63)
    assert wl.total_tokens == 4466
    wl.weights = [wl.weights[0], W.draw_parallel_block_weights(np.random.default_rng(63), wl.dims)]
    for weights in (wl.weights, wl.weights[::-1]):                      # the last block, whose product is sliced, in both forms
        wl.weights = weights
        ctx = context(B, wl, flags, 0.3 if sparse else None)
        want = run(B, wl, ctx, with_geometry=False)
        assert bool(want.isfinite().all())
        tok, cond = B.bits_to_cuda_bf16(wl.packed_tokens()), B.bits_to_cuda_bf16(wl.cond)
        graph, replayed = torch.cuda.CUDAGraph(), torch.empty_like(want)
        with torch.cuda.graph(graph):
            ctx.dit_step_forward(tok, wl.token_lens, cond, 2, out=replayed)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(replayed, want)
        del graph
        host = torch.empty(want.shape, dtype=torch.float32).pin_memory()
        pin = lambda bits: torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).view(torch.bfloat16).pin_memory()
        for _ in range(2):
            host.fill_(float("nan"))
            ctx.dit_step_forward_host(pin(wl.packed_tokens()), wl.token_lens, pin(wl.cond), 2, host)
            assert torch.equal(host, want.cpu())
        ctx.close()


def test_block_scales_hold_where_a_loud_channel_takes_the_row_scales_bits(B):
    """A GELU output channel of 3e4 beside others of a quarter of a unit, into a row of zeros of the down-projection: the exact block does not know
    of it.  Row scales lose the quiet channels' bits to it, block scales those of its own 128 (the oracles of the two modes put the
    blocks' errors at 9.8e-3 and 4.5e-3 of the output, and at 3.6e-3 each without it)."""
    off = {}
    for loud in (0.0, 3e4):
        wl = W.make_custom("loud", W.SMALL, 1, [(128, 128, 13)], seed=64)
        bits = wl.weights[0]
        if loud:
            bits["b_fc1"], bits["w_fc2"] = bits["b_fc1"].copy(), bits["w_fc2"].copy()
            bits["b_fc1"][7], bits["w_fc2"][7] = W.f32_to_bf16_bits(np.float32([loud]))[0], 0
        x, c = W.bf16_to_f64(wl.tokens[0]), W.bf16_to_f64(wl.cond[0])
        exact = O.block_forward(x, c, f64(bits), wl.dims.n_heads, wl.dims.ln_eps)
        for flag in (B.DIT_FLAG_FP8_GEMM, B.DIT_FLAG_FP8_BLOCK128):
            ctx = context(B, wl, flag)
            off[loud, flag] = rms(run(B, wl, ctx).double().cpu().numpy() - exact) / rms(exact)
            ctx.close()
    print(off)
    assert abs(off[0.0, B.DIT_FLAG_FP8_GEMM] - off[0.0, B.DIT_FLAG_FP8_BLOCK128]) <= 0.2 * off[0.0, B.DIT_FLAG_FP8_GEMM]
    assert off[3e4, B.DIT_FLAG_FP8_BLOCK128] <= 0.6 * off[3e4, B.DIT_FLAG_FP8_GEMM]


def test_a_steps_attention_clamps_what_its_sums_carry_beyond_fp32(B):
    """A value channel at 3e38: the weighted sum, taken before the division, is infinite.  The operator would write an infinity, a step the largest
    finite value, like every activation of it (further on an infinity would meet zeros)."""
    import torch
    wl = W.make_custom("clamp", W.SMALL, 1, [(384, 384, 77), (64, 64, 0)], seed=65)
    H = wl.dims.hidden
    wl.weights[0]["b_qkv"] = wl.weights[0]["b_qkv"].copy()
    wl.weights[0]["b_qkv"][2 * H + 5] = W.f32_to_bf16_bits(np.float32([3e38]))[0]
    ctx = context(B, wl, B.DIT_FLAG_SPARSE_ATTENTION | B.DIT_FLAG_BF16_OPERANDS, 0.5)
    run(B, wl, ctx)
    attn, rows = ctx.dit_debug_tap("attn"), wl.token_lens[0]
    ctx.close()
    assert bool(attn.isfinite().all()) and bool((attn[:rows, 5].float() >= 2.9e38).all())

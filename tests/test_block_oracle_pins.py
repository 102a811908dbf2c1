"""Pins of oracle/block_oracle.py: what the reduced forms have to be where the answer is known otherwise."""
import numpy as np
import pytest

from oracle import block_oracle as K
from oracle import dit_oracle as O
from paper_2510_01565_b200 import workloads as W


def test_operands_on_the_grid_multiply_exactly():
    rng = np.random.default_rng(0)
    grid = lambda *s: O.quantize_e4m3(rng.normal(size=s) * 50)
    x, w, b = grid(5, 300), grid(300, 140), rng.normal(size=140)
    x[:, ::128], w[::128, :] = 448.0, 448.0                   # every group's largest value: the scales are 1
    assert np.array_equal(K.block_linear(x, w, b), x @ w + b)
    # and powers of two per group pass through the scales
    sx = 2.0 ** rng.integers(-20, 20, size=(5, 3))
    y = x * np.repeat(sx, 128, axis=1)[:, :300]
    codes, scales = K.quantize_rows(y)
    assert np.array_equal(codes, x) and np.array_equal(scales.T, sx.astype(np.float32))


def test_quantised_values_are_within_half_a_step():
    rng = np.random.default_rng(1)
    x = (rng.normal(size=(7, 257)) * np.exp(rng.normal(size=(7, 1)) * 5)).astype(np.float32)
    codes, scales = K.quantize_rows(x)
    s = np.repeat(scales.astype(np.float64), 128, axis=0)[:257].T
    # normal codes: half of 2^-3 of the leading bit; below 2^-6 half of 2^-9; plus the roundings of the fp32 ratio
    assert np.all(np.abs(codes * s - x) <= np.maximum(np.abs(x) * 2.0 ** -4, s * 2.0 ** -10) * (1 + 2.0 ** -20))
    z, sz = K.quantize_rows(np.zeros((2, 130)))
    assert not z.any() and np.all(sz == np.float32(2.0 ** -100) / np.float32(448))


def test_a_loud_channel_costs_its_own_group_only():
    rng = np.random.default_rng(2)
    x = rng.normal(size=(16, 512))
    quiet = K.quantize_rows(x)
    x[:, 5] *= 4000.0
    loud = K.quantize_rows(x)
    assert np.array_equal(quiet[0][:, 128:], loud[0][:, 128:]) and np.array_equal(quiet[1][1:], loud[1][1:])


@pytest.mark.parametrize("n", [1, 128, 300])
def test_keeping_everything_is_dense_attention(n):
    rng = np.random.default_rng(3)
    q, k, v = (rng.normal(size=(n, 64)) for _ in range(3))
    lists = K.select_blocks(q, k, 2, 99)
    assert lists == [[list(range(-(-n // 128)))] * -(-n // 128)] * 2
    np.testing.assert_allclose(K.sparse_attention(q, k, v, 2, lists), O.attention(q, k, v, 2), rtol=1e-12, atol=1e-12)


def test_selection_by_hand():
    q = np.ones((130, 2))
    k = np.repeat(np.array([[1.0, 1.0], [3.0, 0.0], [0.0, 3.0], [-9.0, 0.0]]), 128, axis=0)[:-100]     # the last block is short
    assert K.select_blocks(q, k, 1, 2) == [[[1, 2], [1, 2]]]            # equal scores 3, 3, then 2
    assert K.select_blocks(q, k, 1, 1) == [[[1], [1]]]                  # the lower of equals
    assert K.select_blocks(q, k, 1, 2, tail=5) == [[[1, 3], [1, 3]]]    # the tail before every score
    assert K.select_blocks(q, k, 1, 2, tail=29) == [[[2, 3], [2, 3]]]   # 28 rows in the last block: one in the block before
    assert K.select_blocks(q, k, 1, 1, tail=29) == [[[2], [2]]]


def test_the_reduced_block_is_the_exact_one_where_nothing_is_reduced():
    wl = W.make_custom("pin", W.SMALL, 1, [(64, 64, 5)], seed=4)
    w = {n: W.bf16_to_f64(t) for n, t in wl.weights[0].items()}
    x, c = W.bf16_to_f64(wl.tokens[0]), W.bf16_to_f64(wl.cond[0])
    exact = O.block_forward(x, c, w, wl.dims.n_heads, wl.dims.ln_eps)
    np.testing.assert_allclose(K.block_forward(x, c, w, wl.dims.n_heads, wl.dims.ln_eps, quantise=False, keep=9), exact, rtol=1e-10, atol=1e-10)
    rms = np.sqrt(np.mean((K.block_forward(x, c, w, wl.dims.n_heads, wl.dims.ln_eps) - exact) ** 2) / np.mean(exact ** 2))
    assert 1e-4 < rms < 1e-1


def test_where_block_scales_are_worth_more_than_row_scales():
    """A down-projection whose operand has one channel that is much louder than the others and multiplies a row of zeros, so that the exact product
    does not know of it.  With one scale for the whole row the others keep e4m3's three bits while they lie above 2^-6 / 448 = 1 / 28672 of
    the largest value; below, its steps of 1 / 229376 of the largest grow against them.  With a scale per 128 columns that happens in one group of
    twelve.  A value of a third of a unit has its last normal step at a loudness of 1e4: there the two begin to part."""
    rng = np.random.default_rng(5)
    u, w = 0.33 * rng.normal(size=(60, 1536)), 0.02 * rng.normal(size=(1536, 384))
    w[7] = 0.0
    off = {}
    for loud in (0.0, 1e3, 3e4):
        u[:, 7] = loud
        y = u @ w
        off[loud] = [float(np.sqrt(np.mean((lin(u, w, 0.0) - y) ** 2) / np.mean(y ** 2))) for lin in (O.fp8_linear, K.block_linear)]
    for loud in (0.0, 1e3):                                             # the same three bits in both
        assert abs(off[loud][0] - off[loud][1]) <= 0.1 * off[loud][1]
    # steps of 3e4 / 229376 = 0.13 for values of 0.33: an error of 0.13 / sqrt(12) = 0.038, 0.11 of them, against e4m3's own 0.036
    assert 0.08 <= off[3e4][0] <= 0.16 and off[3e4][1] <= 0.06

"""Pins of oracle/prompt_oracle.py: hand-computed cases and independent statements."""
import numpy as np

from oracle import prompt_oracle as P


def test_nearest_codes_at_the_borders():
    y = np.array([0, 0.25, 0.2500001, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 5.0001, 6.0, 9.0, -0.25, -0.3, -5.0])
    assert P.nearest_code(y).tolist() == [0, 0, 1, 2, 2, 4, 4, 6, 6, 7, 7, 7, 8, 9, 14]


def test_smallest_exponent():
    top = np.array([6.0, 6.0000001, 3.0, 5.9, 12.0, 2.0 ** -100])
    e = P.exponent_for(top, 6.0)
    assert e.tolist() == [0, 1, -1, 0, 1, -102]
    assert P.exponent_for(np.array([2688.0, 2688.001, 1344.0]), 2688.0).tolist() == [0, 1, -1]


def test_groups_of_32_by_hand():
    x = np.zeros((1, 33))
    x[0, :4], x[0, 32] = [12.0, 1.0, -2.4, 0.4], 0.7
    codes, scales, rows = P.quantize(x, 32)
    assert scales.tolist() == [[2.0, 0.125]] and rows is None
    assert P.values(codes, scales, rows, 32)[0, [0, 1, 2, 3, 32]].tolist() == [12.0, 1.0, -2.0, 0.0, 0.75]      # 0.2 is nearer to 0, 5.6 to 6


def test_groups_of_16_by_hand():
    x = np.zeros((1, 32))
    x[0, 0], x[0, 16], x[0, 17] = 2688.0, 6.0, 2.6
    codes, scales, rows = P.quantize(x, 16)
    assert rows.tolist() == [1.0] and scales.tolist() == [[448.0, 1.0]]
    assert P.values(codes, scales, rows, 16)[0, [0, 16, 17]].tolist() == [2688.0, 6.0, 3.0]
    x[0, 16], x[0, 17] = 2.0 ** -9, 0.0                       # a 2^-20th of the row: its scale is zero
    codes, scales, rows = P.quantize(x, 16)
    assert scales[0, 1] == 0 and not codes[0, 16:].any()


def test_packing_and_scale_tiles():
    assert P.pack(np.array([[1, 2, 15]], np.uint8)).tolist() == [[0x21, 0x0F]]
    scales = np.ones((130, 5))
    scales[33, 4], scales[129, 2] = 2.0, 0.5
    t = P.scale_tiles(scales, 32)
    assert t.shape == (2, 2, 512)
    assert t[0, 1, 1 * 16 + 1 * 4 + 0] == 128 and t[1, 0, 1 * 16 + 0 * 4 + 2] == 126 and t[0, 0, 0] == 127 and t[1, 0, 2 * 16] == 0
    e4m3 = P.scale_tiles(np.array([[448.0, 1.0, 2.0 ** -9, 0.0, 1.875, 2.0 ** -6]]), 16)
    assert e4m3[0, 0, :4].tolist() == [0x7E, 0x38, 0x01, 0x00] and e4m3[0, 1, :2].tolist() == [0x3F, 0x08]


def test_quantisation_error_is_bounded_by_the_widest_step():
    x = np.random.default_rng(0).standard_normal((40, 200)) * np.exp(np.random.default_rng(1).standard_normal((40, 1)))
    for group in (16, 32):
        codes, scales, rows = P.quantize(x, group)
        full = np.repeat(scales, group, axis=1)[:, :200] * (1.0 if rows is None else rows[:, None])
        assert (np.abs(P.values(codes, scales, rows, group) - x) <= full * 1.0001).all()          # half of the step from 4 to 6, and 6.4 clamped


def test_rotation_by_hand():
    x = np.array([[1.0, 0.0, 0.0, 1.0]])
    f = P.frequencies(4)
    assert np.allclose(f, [1.0, 0.01])
    half = P.rotary(x, [1], 1, f)                             # pairs (0, 2) and (1, 3)
    assert np.allclose(half, [[np.cos(1), -np.sin(0.01), np.sin(1), np.cos(0.01)]])
    near = P.rotary(x, [1], 1, f, interleaved=True)           # pairs (0, 1) and (2, 3)
    assert np.allclose(near, [[np.cos(1), np.sin(1), -np.sin(0.01), np.cos(0.01)]])


def test_products_of_rotated_rows_depend_on_their_distance():
    g = np.random.default_rng(2)
    q, k = g.standard_normal((1, 64)), g.standard_normal((1, 64))
    f = P.frequencies(64, factor=4.0, ramp=(1, 8, 512))
    at = lambda i, j: (P.rotary(q, [i], 1, f) @ P.rotary(k, [j], 1, f).T).item()
    assert abs(at(100, 40) - at(1060, 1000)) < 1e-11
    back = P.rotary(P.rotary(q, [77], 1, f), [77], 1, f, inverse=True)
    assert np.allclose(back, q, atol=1e-13)


def test_scaled_frequencies():
    f, s = P.frequencies(8), P.frequencies(8, factor=2.0, ramp=(1.0, 100.0, 2 * np.pi * 10))
    turns = 10 * f                                            # 10, 1, 0.1, 0.01
    assert np.isclose(s[0], f[0] * (9 / 99 + 90 / 99 / 2)) and np.allclose(s[1:], f[1:] / 2) and np.allclose(turns, [10, 1, 0.1, 0.01])
    assert np.allclose(P.frequencies(8, factor=2.0), f / 2)


def test_attention_against_a_masked_softmax():
    g = np.random.default_rng(3)
    q, k, v = g.standard_normal((9, 4 * 8)), g.standard_normal((12, 2 * 8)), g.standard_normal((12, 2 * 8))
    out = P.attention(q, k, v, [4, 5], [4, 8], 4, 2)
    for h in range(4):
        s = q[4:, h * 8:h * 8 + 8] @ k[4:, h // 2 * 8:h // 2 * 8 + 8].T / np.sqrt(8)
        s[np.triu_indices(5, 4, 8)] = -np.inf                 # row i sees keys up to 3 + i
        p = np.exp(s - s.max(1, keepdims=True))
        assert np.allclose(out[4:, h * 8:h * 8 + 8], p / p.sum(1, keepdims=True) @ v[4:, h // 2 * 8:h // 2 * 8 + 8])
    assert np.allclose(out[0], np.concatenate([v[0, :8], v[0, :8], v[0, 8:], v[0, 8:]]))          # the first row sees itself alone
    none = P.attention(q[:3], k[:1], v[:1], [3], [1], 4, 2)
    assert not none[:2].any() and np.allclose(none[2, :8], v[0, :8])

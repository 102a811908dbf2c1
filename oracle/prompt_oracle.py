"""CPU oracle of the operators around a prompt encoder's layer: microscaled 4-bit products, rotary positions, attention over
packed prompts with grouped heads (TEST INFRASTRUCTURE, not a product path; NumPy, shares nothing with the CUDA path).

Everything is fp64; the only fp32 numbers are the two quotients by which the quantiser decides (a scale, a code), which are part of its
definition.
"""
from __future__ import annotations

import numpy as np

from oracle import dit_oracle as O

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
FLOOR = 2.0 ** -100


def nearest_code(y: np.ndarray) -> np.ndarray:
    """Codes 0 .. 15 of the nearest levels to y (fp64), ties to the even code, clamped; 8 marks a negative number."""
    a = np.minimum(np.abs(y), 6.0)
    low = np.clip(np.searchsorted(LEVELS, a, side="right") - 1, 0, 7)
    high = np.minimum(low + 1, 7)
    down, up = a - LEVELS[low], LEVELS[high] - a
    code = np.where((up < down) | ((up == down) & (low % 2 == 1)), high, low)
    return (code + 8 * np.signbit(y)).astype(np.uint8)


def exponent_for(top: np.ndarray, limit: float) -> np.ndarray:
    """Smallest integer e with top <= limit * 2^e."""
    mantissa, e = np.frexp(top / limit)           # (a factor of 6 or 2688 is taken off in fp64: comparisons of 24-bit numbers stay exact)
    e = np.where(mantissa == 0.5, e - 1, e)
    e = np.where(top > limit * np.exp2(e.astype(float)), e + 1, e)
    return np.where(top <= limit * np.exp2(e - 1.0), e - 1, e)


def quantize(x: np.ndarray, group: int):
    """[rows, cols] -> (codes [rows, cols] 0 .. 15, scales [rows, groups], row scales [rows] or None)."""
    rows, cols = x.shape
    x = x.astype(np.float64)
    n = -(-cols // group)
    parts = np.zeros((rows, n * group))
    parts[:, :cols] = x
    parts = parts.reshape(rows, n, group)
    top = np.abs(parts).max(axis=2)
    if group == 32:
        e = exponent_for(np.maximum(top, FLOOR), 6.0)
        scales, row_scales = np.exp2(e.astype(float)), None
        y = parts / scales[:, :, None]
    else:
        e = exponent_for(np.maximum(top.max(axis=1), FLOOR), 6.0 * 448.0)
        row_scales = np.exp2(e.astype(float))
        want = ((top / row_scales[:, None]).astype(np.float32) / np.float32(6.0)).astype(np.float64)
        scales = O.quantize_e4m3(want)
        with np.errstate(divide="ignore", invalid="ignore"):
            y = ((parts / row_scales[:, None, None]).astype(np.float32) / scales[:, :, None].astype(np.float32)).astype(np.float64)
        y = np.where(scales[:, :, None] > 0, y, 0.0)
    return nearest_code(y).reshape(rows, -1)[:, :cols], scales, row_scales


def values(codes: np.ndarray, scales: np.ndarray, row_scales, group: int) -> np.ndarray:
    """What codes and scales stand for, fp64."""
    v = LEVELS[codes & 7] * np.where(codes & 8, -1.0, 1.0) * np.repeat(scales, group, axis=1)[:, :codes.shape[1]]
    return v if row_scales is None else v * row_scales[:, None]


def pack(codes: np.ndarray) -> np.ndarray:
    """Two codes to a byte, the even column in the low half."""
    even = np.zeros((codes.shape[0], -(-codes.shape[1] // 2) * 2), np.uint8)
    even[:, :codes.shape[1]] = codes
    return even[:, 0::2] | even[:, 1::2] << 4


def scale_tiles(scales: np.ndarray, group: int) -> np.ndarray:
    """Scale bytes in tiles of 128 rows x 4 groups: [ceil(rows / 128), ceil(groups / 4), 512], zeros where there is nothing."""
    rows, n = scales.shape
    if group == 32:
        byte = (np.log2(scales) + 127.0).round().astype(np.uint8)
    else:
        mantissa, e = np.frexp(scales)
        byte = np.where(scales >= 2.0 ** -6, ((e + 6) * 8 + mantissa * 16 - 8), scales * 512).round().astype(np.uint8)
    full = np.zeros((-(-rows // 128) * 128, -(-n // 4) * 4), np.uint8)
    full[:rows, :n] = byte
    return full.reshape(-1, 4, 32, full.shape[1] // 4, 4).transpose(0, 3, 2, 1, 4).reshape(full.shape[0] // 128, -1, 512)


def linear(h: np.ndarray, w: np.ndarray, group: int) -> np.ndarray:
    """h w with both operands quantised."""
    a, b = quantize(h, group), quantize(w.T, group)
    return values(*a, group) @ values(*b, group).T


def frequencies(rotary_dim: int, base: float = 10000.0, factor: float = 1.0, ramp=None) -> np.ndarray:
    f = base ** (-np.arange(0, rotary_dim, 2) / rotary_dim)
    if ramp is None:
        return f / factor
    low, high, trained = ramp
    keep = np.clip((trained * f / (2.0 * np.pi) - low) / (high - low), 0.0, 1.0)
    return f * (keep + (1.0 - keep) / factor)


def rotary(x: np.ndarray, positions, n_heads: int, freq: np.ndarray, interleaved: bool = False, magnitude: float = 1.0, inverse: bool = False) -> np.ndarray:
    """x [rows, n_heads * d]: each channel pair as a complex number times magnitude * exp(i position frequency)."""
    y = x.astype(np.float64).reshape(x.shape[0], n_heads, -1).copy()
    turn = magnitude * np.exp((-1j if inverse else 1j) * np.asarray(positions, np.float64)[:, None] * freq)[:, None, :]
    n = len(freq)
    ia, ib = (np.arange(0, 2 * n, 2), np.arange(1, 2 * n, 2)) if interleaved else (np.arange(n), np.arange(n, 2 * n))
    z = (y[:, :, ia] + 1j * y[:, :, ib]) * turn
    y[:, :, ia], y[:, :, ib] = z.real, z.imag
    return y.reshape(x.shape)


def attention(q, k, v, q_lens, kv_lens, n_heads: int, n_kv_heads: int, causal: bool = True, scale: float = 0.0) -> np.ndarray:
    """Row i of a request sees its keys j <= kv_len - q_len + i (all of them without `causal`); a row without keys gives zeros."""
    d = q.shape[1] // n_heads
    scale = scale or 1.0 / np.sqrt(d)
    out = np.zeros(q.shape)
    q0 = k0 = 0
    for lq, lk in zip(q_lens, kv_lens):
        last = lk - lq + np.arange(lq) if causal else np.full(lq, lk - 1)
        seen = np.arange(lk)[None, :] <= last[:, None]
        for h in range(n_heads):
            g = h // (n_heads // n_kv_heads)
            qq = q[q0:q0 + lq, h * d:(h + 1) * d].astype(np.float64)
            kk, vv = (m[k0:k0 + lk, g * d:(g + 1) * d].astype(np.float64) for m in (k, v))
            for i in range(lq):
                n = int(seen[i].sum())
                if n:
                    s = scale * (kk[:n] @ qq[i])
                    p = np.exp(s - s.max())
                    out[q0 + i, h * d:(h + 1) * d] = (p / p.sum()) @ vv[:n]
        q0, k0 = q0 + lq, k0 + lk
    return out

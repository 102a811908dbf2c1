"""CPU oracle of the reduced forms of a block: e4m3 products with one scale per block of 128, and attention over
selected key blocks (TEST INFRASTRUCTURE, not a product path; NumPy, shares nothing with the CUDA path).

Quantisation is a function of fp32 numbers (a maximum, two divisions, a product, one rounding to e4m3), so it is done in
fp32 here as well and its codes are exact; everything else is fp64.  The reference system serves its models in 16-bit
floating point with dense attention (Section 6.1); both forms are approximations of that block with bars of their own.
"""
from __future__ import annotations

import numpy as np

from oracle import dit_oracle as O

BLOCK = 128
FLOOR = np.float32(2.0 ** -100)


def _codes(groups: np.ndarray, top: np.ndarray):
    """groups fp32 with their maxima `top` (broadcastable): code values (fp64) and scales (fp32)."""
    top = np.maximum(top.astype(np.float32), FLOOR)
    ratio = np.float32(448.0) / top
    return O.quantize_e4m3((groups * ratio).astype(np.float32).astype(np.float64)), top / np.float32(448.0)


def quantize_rows(x: np.ndarray):
    """[M, K] -> (codes [M, K], scales [ceil(K / 128), M]): groups of 128 columns of a row."""
    m, k = x.shape
    g = np.zeros((m, -(-k // BLOCK) * BLOCK), np.float32)
    g[:, :k] = x.astype(np.float32)
    g = g.reshape(m, -1, BLOCK)
    codes, scales = _codes(g, np.abs(g).max(axis=2, keepdims=True))
    return codes.reshape(m, -1)[:, :k], scales[:, :, 0].T


def quantize_weight(w: np.ndarray):
    """[K, N] -> (codes [N, K], scales [ceil(N / 128), ceil(K / 128)]): blocks of 128 x 128."""
    k, n = w.shape
    g = np.zeros((-(-n // BLOCK) * BLOCK, -(-k // BLOCK) * BLOCK), np.float32)
    g[:n, :k] = w.T.astype(np.float32)
    g = g.reshape(g.shape[0] // BLOCK, BLOCK, -1, BLOCK)
    codes, scales = _codes(g, np.abs(g).max(axis=(1, 3), keepdims=True))
    return codes.reshape(g.shape[0] * BLOCK, -1)[:n, :k], scales[:, 0, :, 0]


def block_linear(h: np.ndarray, w: np.ndarray, b: np.ndarray) -> np.ndarray:
    """h W + b with both operands quantised in blocks of 128."""
    a, sa = quantize_rows(h)
    c, sc = quantize_weight(w)
    a = a * np.repeat(sa.astype(np.float64), BLOCK, axis=0)[:h.shape[1]].T
    c = c * np.repeat(np.repeat(sc.astype(np.float64), BLOCK, axis=0), BLOCK, axis=1)[:w.shape[1], :w.shape[0]]
    return a @ c.T + b


def select_blocks(q: np.ndarray, k: np.ndarray, n_heads: int, keep: int, tail: int = 0):
    """Per head and query block the ascending list of the `keep` key blocks with the largest product of means."""
    d = q.shape[1] // n_heads
    n = k.shape[0]
    cut = range(0, n, BLOCK)
    lists = []
    for h in range(n_heads):
        c = slice(h * d, (h + 1) * d)
        km = [k[j:j + BLOCK, c].mean(axis=0) for j in cut]
        mine = []
        for i in range(0, q.shape[0], BLOCK):
            qm = q[i:i + BLOCK, c].mean(axis=0)
            score = [np.inf if tail > 0 and j + BLOCK > n - tail else qm @ m for j, m in zip(cut, km)]
            mine.append(sorted(sorted(range(len(km)), key=lambda j: (-score[j], j))[:keep]))
        lists.append(mine)
    return lists


def sparse_attention(q: np.ndarray, k: np.ndarray, v: np.ndarray, n_heads: int, lists) -> np.ndarray:
    """Softmax attention of every query block over its listed key blocks."""
    d = q.shape[1] // n_heads
    out = np.zeros_like(q)
    for h in range(n_heads):
        c = slice(h * d, (h + 1) * d)
        for i, chosen in enumerate(lists[h]):
            rows = slice(i * BLOCK, (i + 1) * BLOCK)
            keys = np.concatenate([np.arange(j * BLOCK, min(len(k), (j + 1) * BLOCK)) for j in chosen])
            out[rows, c] = O.softmax_rows(q[rows, c] @ k[keys, c].T / np.sqrt(d)) @ v[keys, c]
    return out


def block_forward(x: np.ndarray, cond: np.ndarray, w, n_heads: int, eps: float, quantise: bool = True, keep: int | None = None,
                  tail: int = 0) -> np.ndarray:
    """A sequential or parallel adaLN-Zero block with its products through block_linear and its attention over `keep` blocks."""
    H = x.shape[1]
    lin = block_linear if quantise else (lambda a, ww, bb: a @ ww + bb)

    def attend(qkv):
        q, k, v = qkv[:, :H], qkv[:, H:2 * H], qkv[:, 2 * H:]
        if keep is None:
            return O.attention(q, k, v, n_heads)
        return sparse_attention(q, k, v, n_heads, select_blocks(q, k, n_heads, keep, tail))
    if "w_out" in w:
        shift, scale, gate = np.split(O.silu(cond) @ w["w_ada"] + w["b_ada"], 3)
        h = O.modulate(O.layer_norm(x, eps), shift, scale)
        a = attend(lin(h, w["w_qkv"], w["b_qkv"]))
        u = O.gelu_tanh(lin(h, w["w_fc1"], w["b_fc1"]))
        return x + gate * lin(np.concatenate([a, u], axis=1), w["w_out"], w["b_out"])
    shift_a, scale_a, gate_a, shift_m, scale_m, gate_m = O.adaln_modulation(cond, w["w_ada"], w["b_ada"])
    a = attend(lin(O.modulate(O.layer_norm(x, eps), shift_a, scale_a), w["w_qkv"], w["b_qkv"]))
    x = x + gate_a * lin(a, w["w_o"], w["b_o"])
    u = O.gelu_tanh(lin(O.modulate(O.layer_norm(x, eps), shift_m, scale_m), w["w_fc1"], w["b_fc1"]))
    return x + gate_m * lin(u, w["w_fc2"], w["b_fc2"])

"""Whole prompts and caches in 4 or 8 bits in fp64 on the CPU: the format from its list of values, the attention one query after the other.
Shares no code with the GPU path."""
from __future__ import annotations

import math

import numpy as np

LARGEST = {4: 2, 8: 8}            # exponent of the largest value


def grid(bits: int) -> np.ndarray:
    """The magnitudes of the element type, by code."""
    if bits == 4:
        return np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
    return np.array([m / 512 for m in range(8)] + [(1 + m / 8) * 2.0 ** e for e in range(-6, 9) for m in range(8)][:-1])


def quantise(x: np.ndarray, bits: int):
    """Rows (n, d) -> (codes (n, d) one a byte, scale bytes (n, d / 32))."""
    x = np.asarray(x, dtype=np.float64)
    n, d = x.shape
    g = x.reshape(n, d // 32, 32)
    v = grid(bits)
    codes, scales = np.zeros(g.shape, dtype=np.uint8), np.zeros((n, d // 32), dtype=np.uint8)
    for i in range(n):
        for j in range(d // 32):
            top = np.abs(g[i, j]).max()
            if not np.isfinite(g[i, j]).all():
                scales[i, j] = 255
                continue
            e = -1000 if top == 0 else math.frexp(top)[1] - 1
            if top > 1.75 * 2.0 ** e:
                e += 1
            s = min(max(e - LARGEST[bits], -127), 127 - LARGEST[bits])
            y = np.minimum(np.abs(g[i, j]) / 2.0 ** s, v[-1])
            hi = np.searchsorted(v, y)
            lo = np.maximum(hi - 1, 0)
            near = np.where((y - v[lo] < v[hi] - y) | ((y - v[lo] == v[hi] - y) & (lo % 2 == 0)), lo, hi)
            codes[i, j] = near + np.signbit(g[i, j]) * (8 if bits == 4 else 128)
            scales[i, j] = s + 127
    return codes.reshape(n, d), scales


def values(codes: np.ndarray, scales: np.ndarray, bits: int) -> np.ndarray:
    """The way back: what codes (n, d) one a byte and scale bytes (n, d / 32) stand for."""
    v = grid(bits) if bits == 4 else np.append(grid(bits), np.nan)
    table = np.concatenate([v, -v])
    unit = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return table[codes] * np.repeat(unit, 32, axis=1)


def pack(codes: np.ndarray, bits: int) -> np.ndarray:
    return codes if bits == 8 else codes[..., 0::2] | codes[..., 1::2] << 4


def unpack(packed: np.ndarray, bits: int) -> np.ndarray:
    return packed if bits == 8 else np.stack([packed & 15, packed >> 4], axis=-1).reshape(*packed.shape[:-1], -1)


def prompt_attention(q, k, v, H: int, H_kv: int, causal: bool, queries=None):
    """One sequence: q (n_q, H d_k), k and v (n_k, H_kv d_k).  `queries`: those that are computed (None: all).  Returns (out, spread, size, swing), the last
    three for error bounds: spread = sum_j P |v_j - out|, size = sum_j P |v_j| per element, swing = the largest sum |q k| / sqrt(d_k) of a query and head."""
    q, k, v = (np.asarray(x, dtype=np.float64) for x in (q, k, v))
    n_q, n_k, d_k = q.shape[0], k.shape[0], q.shape[1] // H
    out, spread, size, swing = np.zeros(q.shape), np.zeros(q.shape), np.zeros(q.shape), np.zeros((n_q, H))
    for i in range(n_q) if queries is None else queries:
        seen = min(i + n_k - n_q + 1, n_k) if causal else n_k
        if seen <= 0:
            continue
        for h in range(H):
            c, ck = slice(h * d_k, (h + 1) * d_k), slice(h * H_kv // H * d_k, (h * H_kv // H + 1) * d_k)
            s = k[:seen, ck] @ q[i, c] / math.sqrt(d_k)
            swing[i, h] = (np.abs(k[:seen, ck]) @ np.abs(q[i, c])).max() / math.sqrt(d_k)
            p = np.exp(s - s.max())
            p /= p.sum()
            out[i, c] = p @ v[:seen, ck]
            spread[i, c] = p @ np.abs(v[:seen, ck] - out[i, c])
            size[i, c] = p @ np.abs(v[:seen, ck])
    return out, spread, size, swing

"""A tree of drafted tokens in fp64 on the CPU: its attention the vanilla way (K and V stored, one node after the other), the walk
that accepts drafted tokens, and the move of the accepted keys.  Shares no code with the GPU path."""
from __future__ import annotations

import math

import numpy as np


def chain(parents, i: int):
    """Node i and its ancestors, or None for an unused slot."""
    out = []
    while True:
        out.append(i)
        up = int(parents[i])
        if up == -1:
            return out
        if up < -1 or up >= i:
            return None
        i = up


def rotate(x: np.ndarray, H: int, pos: np.ndarray, base: float) -> np.ndarray:
    """Rows x (n, d) rotated per head and adjacent pair by their positions: y1 = x1 cos + x2 sin, y2 = x2 cos - x1 sin."""
    n, d = x.shape
    half = d // H // 2
    ang = np.asarray(pos, dtype=np.float64)[:, None] * base ** (-np.arange(half) / half)
    z = x.reshape(n, H, half, 2)
    z = (z[..., 0] + 1j * z[..., 1]) * np.exp(-1j * ang)[:, None, :]
    return np.stack([z.real, z.imag], axis=-1).reshape(n, d)


def tree_attention(q, K, W_KV, parents, length: int, H: int, base=None, nodes=None):
    """q (N, d), K (length + N, d) raw keys, W_KV (d, d), parents (N,).  `nodes`: the nodes that are computed (None: all); the others' rows are 0.  Returns (out (N, d), spread, size, swing), the last three
    for error bounds: spread = sum_t P |V_t - out|, size = (P |K|) |W_KV| per element of the result, swing = the largest
    sum_j |q_j k_tj| / sqrt(d_k) of a node and head over its rows."""
    q, K, W = (np.asarray(x, dtype=np.float64) for x in (q, K, W_KV))
    N, d = q.shape
    d_k = d // H
    out, spread, size, swing = np.zeros((N, d)), np.zeros((N, d)), np.zeros((N, d)), np.zeros((N, H))
    for i in range(N) if nodes is None else nodes:
        seen = chain(parents, i)
        if seen is None:
            continue
        rows = list(range(length)) + [length + j for j in seen]
        pos = list(range(length)) + [length + len(chain(parents, j)) - 1 for j in seen]
        Ki = K[rows]
        key = Ki if base is None else rotate(Ki, H, np.array(pos), base)
        V = Ki @ W
        absW = np.abs(W)
        for h in range(H):
            c = slice(h * d_k, (h + 1) * d_k)
            s = key[:, c] @ q[i, c] / math.sqrt(d_k)
            swing[i, h] = (np.abs(key[:, c]) @ np.abs(q[i, c])).max() / math.sqrt(d_k)
            p = np.exp(s - s.max())
            p /= p.sum()
            out[i, c] = p @ V[:, c]
            spread[i, c] = p @ np.abs(V[:, c] - out[i, c])
            size[i, c] = (p @ np.abs(Ki)) @ absW[:, c]
    return out, spread, size, swing


def verify(tokens, parents, p, draft, u):
    """One sequence: tokens, parents, u (N,), p and draft (N, V) or draft None.  Returns (path, next token): the residual distribution is
    carried along as a vector and normalised after every rejection."""
    N, V = p.shape
    p = np.asarray(p, dtype=np.float64)
    draft = None if draft is None else np.asarray(draft, dtype=np.float64)
    u = np.asarray(u, dtype=np.float64)
    cur, path = 0, [0]
    left, total = p[0].copy(), 1.0
    i = 1
    while i < N:
        x = int(tokens[i])
        if int(parents[i]) == cur and 0 <= x < V:
            q = draft[cur] if draft is not None else None
            if (u[i] * total * q[x] if q is not None else u[i] * total) < left[x]:
                cur = i
                path.append(i)
                left, total = p[i].copy(), 1.0
            elif q is not None:
                left = np.maximum(left - total * q, 0.0)
                total = left.sum()
            else:
                total -= left[x]
                left[x] = 0.0
        i += 1
    run = np.cumsum(left)
    if run[-1] > 0:
        over = np.nonzero(run > u[0] * run[-1])[0]
        nxt = int(over[0]) if len(over) else int(np.nonzero(left > 0)[0][-1])
    else:
        nxt = int(np.argmax(p[cur]))
    return path, nxt


def commit(K, path, length: int):
    """Rows length + path[j] of K (rows, d) to length + j, one after the other."""
    K = K.copy()
    for j, i in enumerate(path):
        K[length + j] = K[length + i]
    return K

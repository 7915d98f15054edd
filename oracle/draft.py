"""Plain float64 / integer definitions of a speculative decoding step's operators.

Rows of a QKV product normalised, rotated and put into a paged cache, attention of
drafted trees over it, sampling, and the move of keys and values between slots,
each written out from its definition.  Nothing here follows the kernels' order of
work.  Bits are bfloat16 storage (uint16); a cache is [pages, 2, nkv, 16 * hd].
"""

from __future__ import annotations

import math

import numpy as np

PAGE = 16


def tile_places(hd: int):
    """Element of (key of the page, dim) within a K tile and within a V^T tile, [16, hd] each."""
    k, v = np.zeros((PAGE, hd), np.int64), np.zeros((PAGE, hd), np.int64)
    for r in range(PAGE):
        for e in range(hd):
            k[r, e] = ((e // 32 * 4 + (e // 8) % 4) * 16 + r) * 8 + e % 8
            v[r, e] = ((e // 32 * 4 + r // 4) * 16 + e % 16) * 8 + ((e // 16) % 2) * 4 + r % 4
    return k, v


def rope_rows(qkv, nq: int, nkv: int, hd: int, q_gain, k_gain, eps: float, rope, pos):
    """qkv [T, (nq + 2 nkv) hd] -> float64 q [T, nq, hd], k, v [T, nkv, hd]; rope [n_pos, hd / 2, 2]."""
    y = np.asarray(qkv, np.float64).reshape(len(qkv), nq + 2 * nkv, hd)
    out = np.empty_like(y)
    for t in range(len(y)):
        p = int(pos[t])
        for h in range(nq + 2 * nkv):
            x = y[t, h]
            if h < nq + nkv:
                gain = q_gain if h < nq else k_gain
                if gain is not None:
                    x = x / math.sqrt(float(np.sum(x * x)) / hd + eps) * gain
                if not 0 <= p < len(rope):
                    x = np.full(hd, np.nan)
                else:
                    c, s = np.asarray(rope[p], np.float64).T
                    a, b = x[:hd // 2], x[hd // 2:]
                    x = np.concatenate([a * c - b * s, a * s + b * c])
            out[t, h] = x
    return out[:, :nq], out[:, nq:nq + nkv], out[:, nq + nkv:]


def kv_move(pool_bits, hd: int, src, dst, offsets):
    """pool_bits [layers, pages, 2, nkv, 16 * hd] after the moves."""
    places = tile_places(hd)
    new = pool_bits.copy()
    slots = pool_bits.shape[1] * PAGE
    for lo, hi in zip(offsets[:-1], offsets[1:]):
        for j in range(lo, hi):
            a, b = int(src[j]), int(dst[j])
            if 0 <= a < slots and 0 <= b < slots:
                for c in range(2):
                    new[:, b // PAGE, c, :, places[c][b % PAGE]] = pool_bits[:, a // PAGE, c, :, places[c][a % PAGE]]
    return new


def tree_attention(q, K, V, see):
    """q [n, nq, hd], K, V [keys, nkv, hd] (float64), see [n, keys] -> [n, nq, hd]; keys a query does not see take no part."""
    n, nq, hd = q.shape
    group = nq // K.shape[1]
    out = np.zeros((n, nq, hd))
    for r in range(n):
        mine = np.flatnonzero(see[r])
        for j in range(nq):
            h = j // group
            z = K[mine, h] @ q[r, j] / math.sqrt(hd)
            if len(z) and np.max(z) != -np.inf:  # (a NaN score makes NaN)
                p = np.exp(z - np.max(z))
                out[r, j] = (p / p.sum()) @ V[mine, h]
    return out


def sample(x, u: float, temperature: float = 1.0, top_k: int = 0, top_p: float = 1.0, min_p: float = 0.0):
    """(token, probability) of one row of logits."""
    x = np.asarray(x, np.float64)
    tokens = np.flatnonzero(x > -np.inf)  # (a NaN is not)
    if len(tokens) == 0:
        return -1, 0.0
    tokens = tokens[np.argsort(-x[tokens], kind="stable")]
    if not temperature > 0:
        return int(tokens[0]), 1.0
    v = x[tokens]
    d = np.zeros(len(v))
    lower = v < v[0]
    d[lower] = np.inf if v[0] == np.inf else (v[0] - v[lower]) / temperature
    w = np.exp(-d)
    w[w < 2.0 ** -46] = 0.0
    if min_p > 0:
        w = w[w >= min(min_p, 1.0)]
    if top_k > 0:
        w = w[:top_k]
    if top_p < 1:
        enough = np.flatnonzero(np.cumsum(w) >= top_p * math.fsum(w))
        w = w[:enough[0] + 1] if len(enough) else w
    w = w[w > 0]
    total = math.fsum(w)
    upto = np.cumsum(w)
    at = int(np.searchsorted(upto, (u if u > 0 else 0.0) * total, side="right"))
    at = len(w) - 1 if u >= 1 else min(at, len(w) - 1)
    return int(tokens[at]), float(w[at] / total)

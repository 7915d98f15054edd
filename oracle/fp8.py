"""Plain float64 / integer definitions of the 8-bit feed-forward operators.

Rows of e4m3 codes with a power of two for each 128 values, the product of such
rows, RMSNorm with the residual's addition, SwiGLU, the router of tokens to
experts and the weighted sum of their rows, each written out from its
definition.  Nothing here follows the kernels' order of work.
"""

from __future__ import annotations

import math

import numpy as np

GROUP = 128
E4M3_MAX = 448.0
MIN_BYTE = 1  # the least power of two is 2^-126
INF_BYTE = 247  # of a group that holds an infinity (the next above the largest finite values')

# value of each of the 256 codes: sign, 4 exponent bits (bias 7), 3 mantissa bits; 0x7f and 0xff are NaN
CODE_VALUES = np.array([(-1.0 if c & 0x80 else 1.0) * (float("nan") if c & 0x7F == 0x7F else
                        (c & 7) * 2.0 ** -9 if c & 0x78 == 0 else
                        (8 + (c & 7)) * 2.0 ** (((c >> 3) & 15) - 10)) for c in range(256)])
_POSITIVE = CODE_VALUES[:0x7F]  # 0 .. 448, ascending


def e4m3_code(v: np.ndarray) -> np.ndarray:
    """Code nearest to each value (|v| <= 448), ties to the even code; not finite: the NaN code."""
    v = np.asarray(v, np.float64)
    finite = np.isfinite(v)
    a = np.abs(np.where(finite, v, 0.0))
    hi = np.clip(np.searchsorted(_POSITIVE, a), 1, 0x7E)  # _POSITIVE[hi - 1] < a <= _POSITIVE[hi]
    lo = hi - 1
    below, above = a - _POSITIVE[lo], _POSITIVE[hi] - a
    code = np.where((above < below) | ((above == below) & (hi % 2 == 0)), hi, lo)
    code = np.where(finite, code, 0x7F)
    return (code + np.where(np.signbit(v), 0x80, 0)).astype(np.uint8)


def group_byte(top: np.ndarray) -> np.ndarray:
    """E8M0 byte of groups whose largest magnitude is `top`: the smallest power of two with top <= 448 * 2^(E - 127)."""
    out = np.full(np.shape(top), MIN_BYTE, np.int64)
    for i, t in np.ndenumerate(np.asarray(top, np.float64)):
        e = MIN_BYTE
        if np.isinf(t):
            e = INF_BYTE
        elif t > 0:
            e = max(e, math.frexp(t / E4M3_MAX)[1] + 127)
            while e > MIN_BYTE and t <= E4M3_MAX * 2.0 ** (e - 1 - 127):
                e -= 1
        out[i] = e
    return out


def grouped(v: np.ndarray) -> np.ndarray:
    """[rows, n] -> [rows, groups, 128], zeros behind n."""
    rows, n = v.shape
    g = -(-n // GROUP)
    out = np.zeros((rows, g * GROUP), np.float64)
    out[:, :n] = v
    return out.reshape(rows, g, GROUP)


def quantise(v: np.ndarray):
    """Values [rows, n] -> codes [rows, 128 * groups], bytes [rows, groups]."""
    q = grouped(np.asarray(v, np.float64))
    top = np.max(np.where(np.isnan(q), 0.0, np.abs(q)), axis=2)
    byte = group_byte(top)
    return e4m3_code(q / 2.0 ** (byte[:, :, None] - 127.0)).reshape(len(v), -1), byte.astype(np.uint8)


def values(codes: np.ndarray, byte: np.ndarray) -> np.ndarray:
    """float64 values of codes [rows, 128 * groups] with bytes [rows, >= groups]."""
    g = codes.shape[1] // GROUP
    return CODE_VALUES[codes] * np.repeat(2.0 ** (byte[:, :g].astype(np.float64) - 127.0), GROUP, axis=1)


def rms_norm(x: np.ndarray, gain: np.ndarray, eps: float) -> np.ndarray:
    x = np.asarray(x, np.float64)
    return x / np.sqrt(np.mean(x * x, axis=1, keepdims=True) + eps) * np.asarray(gain, np.float64)


def swiglu_rows(y: np.ndarray) -> np.ndarray:
    """silu(gate) * up of products whose columns come as 8 gate, then the 8 matching up ones."""
    b = np.asarray(y, np.float64).reshape(len(y), y.shape[1] // 16, 2, 8)
    gate, up = b[:, :, 0], b[:, :, 1]
    return (gate / (1.0 + np.exp(-gate)) * up).reshape(len(y), y.shape[1] // 2)


def route(logits, k: int, bias=None, sigmoid=False, groups=1, top_groups=1, renormalise=True, scale=1.0):
    """(experts [T, k], weights [T, k], offsets [E + 1], src [T * k], slot [T, k]), token by token."""
    logits = np.asarray(logits, np.float64)
    T, E = logits.shape
    per = E // groups
    experts = np.zeros((T, k), np.int64)
    weights = np.zeros((T, k))
    for t in range(T):
        z = logits[t]
        with np.errstate(all="ignore"):
            if sigmoid:
                s = 1.0 / (1.0 + np.exp(-z))
            elif np.all(z == -np.inf):
                s = np.zeros(E)
            else:
                e = np.where(z == -np.inf, 0.0, np.exp(z - np.nanmax(np.concatenate([z, [-np.inf]]))))
                s = e / e.sum()
            c = s + (np.asarray(bias, np.float64) if bias is not None else 0.0)
        c = [v if v == v else -math.inf for v in c]
        best = []
        for g in range(groups):
            open_ = sorted(v for v in c[g * per:(g + 1) * per] if v > -math.inf)
            best.append(sum(open_[-2:]) if open_ else -math.inf)
        kept = sorted(range(groups), key=lambda g: (-best[g], g))[:top_groups]
        left = [e for e in range(E) if e // per in kept]
        experts[t] = sorted(left, key=lambda e: (-c[e], e))[:k]
        shut = [bias is not None and bias[e] == -math.inf for e in range(E)]
        total = sum(s[e] for e in experts[t] if not shut[e])
        for j, e in enumerate(experts[t]):
            weights[t, j] = (0.0 if shut[e] else s[e]) / (total if renormalise and total != 0 else 1.0) * scale
    offsets, src, slot = [0], [], np.zeros((T, k), np.int64)
    for e in range(E):
        for t in range(T):
            for j in range(k):
                if experts[t, j] == e:
                    slot[t, j] = len(src)
                    src.append(t)
        offsets.append(len(src))
    return experts, weights, np.array(offsets), np.array(src, np.int64), slot


def combine(y, weights, slot, resid=None):
    """resid + sum_j weights[t, j] * y[slot[t, j]]; slots outside y add nothing."""
    y, weights = np.asarray(y, np.float64), np.asarray(weights, np.float64)
    T, k = slot.shape
    out = np.zeros((T, y.shape[1])) if resid is None else np.array(resid, np.float64)
    for t in range(T):
        for j in range(k):
            if 0 <= slot[t, j] < len(y):
                out[t] += weights[t, j] * y[slot[t, j]]
    return out


def packed_codes(codes: np.ndarray) -> np.ndarray:
    """Codes [N, Kp] in the products' weight layout, element by element."""
    N, Kp = codes.shape
    n, k = np.meshgrid(np.arange(N), np.arange(Kp), indexing="ij")
    at = ((n // 16 * (Kp // 128) + k // 128) * 2 + k // 64 % 2) * 1024 + (n % 16 + 16 * (k // 16 % 4)) * 16 + k % 16
    out = np.zeros(N * Kp, np.uint8)
    out[at.ravel()] = codes.ravel()
    return out


def packed_bytes(byte: np.ndarray, fill: int = 127) -> np.ndarray:
    """Bytes [N, Kp / 128] in the products' weight layout (`fill` where a last four is not full)."""
    N, B = byte.shape
    G = -(-B // 4) * 4
    out = np.full(N * G, fill, np.uint8)
    n, b = np.meshgrid(np.arange(N), np.arange(B), indexing="ij")
    out[(((n // 16 * (G // 4) + b // 4) * 16 + n % 16) * 4 + b % 4).ravel()] = byte.ravel()
    return out

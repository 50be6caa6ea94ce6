"""CPU oracle of the operators on microscaled 4-bit floating point and of the mixture-of-experts layer (TEST INFRASTRUCTURE,
never the product path).  Plain numpy in 64 bits; imports nothing from the GPU package.

Format: blocks of 32 along the last axis; codes [..., K/2] (even k in the low nibble, bit 3 of a code the sign), scales
[..., K/32], s = 2^(s - 127), 255 = the block is NaN.
"""
from __future__ import annotations

import numpy as np

MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def element(code):
    """The value of a 4-bit code."""
    code = np.asarray(code)
    v = MAGNITUDES[code & 7]
    return np.where(code & 8, -v, v)


def nearest_code(a):
    """The code (0..7) of the element nearest to a >= 0, by exhaustive comparison; ties to the even code, beyond 6 to 6."""
    a = np.asarray(a, np.float64)
    best = np.zeros(a.shape, np.int64)
    dist = np.abs(a - MAGNITUDES[0])
    for c in range(1, 8):
        d = np.abs(a - MAGNITUDES[c])
        better = (d < dist) | ((d == dist) & (c % 2 == 0))
        best = np.where(better, c, best)
        dist = np.where(better, d, dist)
    return best


def quantize(X):
    """X [..., K] float64 holding the input's exact values -> (codes, scales) uint8."""
    X = np.asarray(X, np.float64)
    K = X.shape[-1]
    b = X.reshape(-1, K // 32, 32)
    finite = np.isfinite(b).all(axis=2)
    most = np.where(finite, np.max(np.abs(np.where(np.isfinite(b), b, 0.0)), axis=2), 1.0)
    # frexp: a = f 2^e with f in [1/2, 1), so floor(log2 a) = e - 1
    e = np.where(most > 0, np.frexp(np.where(most > 0, most, 1.0))[1] - 1 - 2, -127)
    e = np.clip(e, -127, 127)
    clean = np.where(finite[:, :, None], b, 0.0)
    q = nearest_code(np.ldexp(np.abs(clean), -e[:, :, None])) + 8 * (np.signbit(clean) & finite[:, :, None])
    q = q.astype(np.uint8).reshape(-1, K)
    codes = q[:, 0::2] | (q[:, 1::2] << 4)
    scales = np.where(finite, e + 127, 255).astype(np.uint8)
    lead = X.shape[:-1]
    return codes.reshape(*lead, K // 2), scales.reshape(*lead, K // 32)


def values(codes, scales):
    """The float64 values [..., K]."""
    codes, scales = np.asarray(codes), np.asarray(scales)
    q = np.stack([codes & 15, codes >> 4], axis=-1).reshape(*codes.shape[:-1], -1)
    s = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(np.int64) - 127))
    return element(q) * np.repeat(s, 32, axis=-1)


def gemm(X, codes, scales):
    """(Y, A) = (X W^T, |X| |W|^T) in 64 bits: the result and the sum of the terms' magnitudes."""
    X = np.asarray(X, np.float64)
    W = values(codes, scales)
    return X @ W.T, np.abs(X) @ np.abs(W).T


def route(logits, top_k, sigmoid=False, renormalize=True, factor=1.0):
    """(ids, weights) one token at a time, from the definition: descending, ties to the lowest index, NaN first, -inf never chosen."""
    logits = np.asarray(logits, np.float64)
    T, E = logits.shape
    ids = np.full((T, top_k), -1, np.int64)
    weights = np.zeros((T, top_k))
    for t in range(T):
        row = logits[t]
        key = np.where(np.isnan(row), np.inf, row)
        order = sorted((e for e in range(E) if row[e] != -np.inf), key=lambda e: (not np.isnan(row[e]), -key[e], e))[:top_k]
        if not order:
            continue
        with np.errstate(all="ignore"):
            if sigmoid:  # by its logarithm, -log(1 + e^-l): quotients of sigmoids that are themselves below the range of 64 bits
                log = -np.logaddexp(0.0, -row[order])
                chosen = np.exp(log - log.max() if renormalize else log)
                total = 1.0
            else:
                score = np.exp(row - row[order[0]])
                total = score.sum()
                chosen = score[order]
            if renormalize:
                total = chosen.sum()
            ids[t, :len(order)] = order
            weights[t, :len(order)] = chosen / total * factor
    return ids, weights


def activate(g, gelu=False):
    with np.errstate(over="ignore"):
        if gelu:
            return 0.5 * g * (1.0 + np.tanh(np.sqrt(2.0 / np.pi) * (g + 0.044715 * g ** 3)))
        return g / (1.0 + np.exp(-g))


def experts(X, ids, weights, W13, W2, gelu=False):
    """Y [T, H] of the layer; W13 [E, 2 I, H] and W2 [E, H, I] are values."""
    X = np.asarray(X, np.float64)
    Y = np.zeros_like(X)
    I = W2.shape[2]
    for t in range(X.shape[0]):
        for j in range(ids.shape[1]):
            e = ids[t, j]
            if 0 <= e < W13.shape[0]:
                both = W13[e] @ X[t]
                Y[t] += weights[t, j] * (W2[e] @ (activate(both[:I], gelu) * both[I:]))
    return Y

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

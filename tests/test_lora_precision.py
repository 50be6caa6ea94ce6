"""Adapters and their gradients: sums that keep FP32's bits until the one rounding, at values where fewer would show.  Every input, product and sum here is exact in FP32 and every
result exact in its type, so results are compared as they are: a value of H or G that loses a bit on its way into the second product changes them.
"""
import numpy as np
import pytest

from test_lora import KINDS, exact, lora  # noqa: F401

gpu = pytest.mark.gpu


def tensor(a, kind):
    import torch
    t = torch.tensor(a, dtype=torch.float64).to(getattr(torch, kind))
    assert torch.equal(t.double(), torch.tensor(a, dtype=torch.float64))
    return t.cuda()


def pairs(M, R, width, other, kind):
    """Rows two by two: `long` [M, width] times `thin` [R, width] is 1 + 2^-9 + j 2^-17 and 1 + 2^-9 in a pair's rows (j = 1, 2, 3 by the column of the result), `wide` [M, other] is v and -v.
    Sums over the rows of their products: j 2^-17 v for each pair, at most 18 2^-17 in all."""
    long, thin, wide = np.zeros((M, width)), np.zeros((R, width)), np.zeros((M, other))
    long[:, 0], long[:, 1], long[0::2, 2] = 1.0, 2.0 ** -9, 2.0 ** -17
    thin[:, 0], thin[:, 1], thin[:, 2] = 1.0, 1.0, 1 + np.arange(R) % 3
    sign = 1.0 - 2.0 * (np.arange(M // 2) % 2)
    sign[-1] = 1.0
    v = np.outer(sign, 1.0 + np.arange(other) % 3)
    wide[0::2], wide[1::2] = v, -v
    return long, thin, wide, np.outer(thin[0:, 2] * 2.0 ** -17, v.sum(0))


@gpu
@pytest.mark.parametrize("grads", ["same", "float32"])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("M,L,R,K,N", [(2, 1, 8, 64, 64), (70, 3, 16, 264, 136), (130, 2, 32, 136, 264), (64, 2, 64, 200, 72), (66, 2, 128, 72, 200), (40, 130, 24, 584, 600)])
def test_gradients_of_rows_that_nearly_cancel(lora, M, L, R, K, N, kind, grads):
    """All rows are of one adapter.  dA from G = dY B, dB from H = X A^T."""
    import torch
    dtype = torch.float32 if grads == "float32" else getattr(torch, kind)
    ids = torch.full((M,), L - 1, dtype=torch.int32, device="cuda")
    dy, b, x, want = pairs(M, R, N, K, kind)
    A, B = torch.zeros(L, R, K, device="cuda").to(getattr(torch, kind)), torch.zeros(L, N, R, device="cuda").to(getattr(torch, kind))
    B[L - 1] = tensor(b.T.copy(), kind)
    _, dA, _ = lora.grad(tensor(dy, kind), tensor(x, kind), A, B, ids, dtype=dtype)
    assert np.array_equal(exact(dA[L - 1]), want) and not exact(dA[:L - 1]).any()
    x, a, dy, want = pairs(M, R, K, N, kind)
    B.zero_()
    A[L - 1] = tensor(a, kind)
    _, _, dB = lora.grad(tensor(dy, kind), tensor(x, kind), A, B, ids, dtype=dtype)
    assert np.array_equal(exact(dB[L - 1]), want.T) and not exact(dB[:L - 1]).any()

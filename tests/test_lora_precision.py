"""Adapters and their gradients: sums that keep FP32's bits until the one rounding, at values where fewer would show.  Where a test names no bound,
every input, product and sum is exact in FP32 and every result exact in its type, so results are compared as they are: a value of H or G that loses a bit on its way into the second product
changes them.
"""
import math

import numpy as np
import pytest

from oracle import grouped_oracle as go
from test_lora import KINDS, compare, exact, expected_add, expected_grad, lora, make  # noqa: F401

gpu = pytest.mark.gpu


def tensor(a, kind):
    import torch
    t = torch.tensor(a, dtype=torch.float64).to(getattr(torch, kind))
    assert np.array_equal(t.double().numpy(), np.asarray(a, dtype=np.float64), equal_nan=True)
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


@gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("R", [8, 16, 32, 64, 72, 128])
@pytest.mark.parametrize("M", [3, 20, 90, 300])
def test_a_row_of_h_far_from_its_largest_value(lora, M, R, kind):
    """H is 2^20 in the first rank and 2^-20 in the last; half of the columns of B have the first alone, the others the last alone.  dX the same with G."""
    import torch
    K, N = 72, 136
    x, a, b, y = np.zeros((M, K)), np.zeros((R, K)), np.zeros((N, R)), np.zeros((M, N))
    x[:, 0], a[0, 0], b[0::2, 0] = 1024.0, 1024.0, 2.0 ** -10
    x[:, 1], a[R - 1, 1], b[1::2, R - 1] = 2.0 ** -10, 2.0 ** -10, 1024.0
    y[:, 1::2] = 2.0 ** -9
    want = np.where(np.arange(N) % 2, 2.0 ** -9 + 2.0 ** -10, 2.0 ** 10)
    ids = torch.zeros(M, dtype=torch.int32, device="cuda")
    out = lora.add(tensor(y, kind), tensor(x, kind), tensor(a[None], kind), tensor(b[None], kind), ids)
    assert np.array_equal(exact(out), np.broadcast_to(want, (M, N)))
    # G = dY B with dY in X's place and B in A's; dX = G A with A in B's
    dX, _, _ = lora.grad(tensor(x, kind), tensor(y, kind), tensor(b.T[None].copy(), kind), tensor(a.T[None].copy(), kind), ids, dX=tensor(y, kind), dtype=torch.float32)
    assert np.array_equal(exact(dX), np.broadcast_to(want, (M, N)))


@gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("R", [8, 40, 128])
@pytest.mark.parametrize("M", [7, 75])
@pytest.mark.parametrize("first,second", [(2.0 ** 12, 2.0 ** -12), (2.0 ** -10, 2.0 ** 6), (1.0, 1.0)])
def test_h_beyond_fp16_on_either_side(lora, M, R, kind, first, second):
    """H and G of about 2^24 (beyond 65504), of 2^-20 (among FP16's numbers of fewer bits) and of ordinary size, random, within the bounds of the other tests."""
    import torch
    L, K, N = 3, 264, 328
    Y, X, A, B, ids, scaling = make(M, L, R, K, N, kind, 11, "mixed")
    X, A, B, Y = X * first, A * first, B * second, Y * second
    assert all(bool(t.isfinite().all()) for t in (X, A, B, Y))
    ref, bound = expected_add(exact(Y), exact(X), exact(A), exact(B), ids, exact(scaling))
    compare(lora.add(Y, X, A, B, ids, scaling), ref, bound, "out")
    # G of the size of H: dY like X, B like A
    B, Y = (B / second * first), (Y / second * first)
    A = A / first * second
    got = lora.grad(Y, X, A, B, ids, scaling, dtype=torch.float32)
    want = expected_grad(exact(Y), exact(X), exact(A), exact(B), ids, exact(scaling), np.zeros((M, K)))
    for g, (r, bnd), name in zip(got, want, ("dX", "dA", "dB")):
        compare(g, r, bnd, name)


@gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("R", [8, 24, 64, 128])
@pytest.mark.parametrize("M", [5, 90])
def test_infinities_of_rows_and_weights_stay_infinities(lora, M, R, kind):
    """Every finite H is 1 and every finite weight of B 1, numbers that are one 16-bit number and zeros."""
    K, N = 64, 136
    x, a, b, y = np.ones((M, K)), np.full((2, R, K), 1 / K), np.ones((2, N, R)), np.ones((M, N))
    x[1, 7], x[4, 0], b[0, 3, 0], b[0, 5, R - 1], b[1, 130, 2] = math.inf, -math.inf, math.inf, -math.inf, math.nan
    ids = np.arange(M) % 2
    ids[2] = -1
    with np.errstate(invalid="ignore"):
        want = go.lora_add(y, x, a, b, ids, [1.0, 1.0])
    assert np.isinf(want).sum() >= 2 * N and np.isfinite(want[2]).all()
    import torch
    who = torch.tensor(ids, dtype=torch.int32, device="cuda")
    args = [tensor(v, kind) for v in (y, x, a, b)]
    np.testing.assert_array_equal(exact(lora.add(*args, who)), want)
    dX, _, _ = lora.grad(args[1], args[0], args[3].transpose(1, 2).contiguous(), args[2].transpose(1, 2).contiguous(), who, dX=args[0])
    np.testing.assert_array_equal(exact(dX), want)


@gpu
@pytest.mark.parametrize("grads", ["same", "float32"])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("R", [8, 24, 64, 128])
@pytest.mark.parametrize("M", [9, 90])
def test_infinities_of_rows_and_gradients_stay_infinities(lora, M, R, kind, grads):
    """Every finite value of G, H, X and dY is 1."""
    import torch
    K, N = 64, 128
    x, dy, a, b = np.ones((M, K)), np.ones((M, N)), np.full((2, R, K), 1 / K), np.full((2, N, R), 1 / N)
    x[1, 7], x[6, 9], dy[4, 0], dy[5, 3] = math.inf, -math.inf, math.inf, math.inf
    ids = np.arange(M) % 2
    ids[5] = -1
    with np.errstate(invalid="ignore"):
        want = go.lora_grad(dy, x, a, b, ids, [1.0, 1.0], np.zeros((M, K)))
    assert all(np.isinf(w).any() for w in want) and np.isfinite(want[1][1][:, :7]).all() and np.isnan(want[1][0][:, 9]).all()
    got = lora.grad(*[tensor(v, kind) for v in (dy, x, a, b)], torch.tensor(ids, dtype=torch.int32, device="cuda"), dtype=torch.float32 if grads == "float32" else getattr(torch, kind))
    for g, w in zip(got, want):
        np.testing.assert_array_equal(exact(g), w)

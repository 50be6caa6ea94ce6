"""Gathered rows of an X on either side of 2 GiB, at sizes that the 256 x 256 tiles are planned for: they take row offsets of 32 bits, and beyond that the 128 x 128 tiles step in.
Tolerances: test_grouped.py."""
import numpy as np
import pytest

from oracle import grouped_oracle as go
from test_grouped import compare, exact, generator, grouped, ints, tolerance, values  # noqa: F401

gpu = pytest.mark.gpu


@gpu
@pytest.mark.parametrize("x_rows", [(1 << 20) - 1, (1 << 20) + 8])
def test_gathered_rows_on_either_side_of_two_gib(grouped, x_rows):
    import torch
    K, N, top_k, sizes = 1024, 8192, 3, [300, 0, 500, 224]
    count, E = sum(sizes), len(sizes)
    assert (x_rows * K * 2 >= 1 << 31) == (x_rows > 1 << 20)
    assert grouped.query_tile(E, count, N, K) == (256, 256) and grouped.query_tile(E, count, N, K, grad=True) == (256, 256)
    gen, rng = generator(21), np.random.default_rng(21)
    X = torch.empty(x_rows, K, device="cuda", dtype=torch.bfloat16)
    for i in range(0, x_rows, 1 << 18):
        X[i:i + (1 << 18)] = values(gen, (min(1 << 18, x_rows - i), K), "bfloat16")
    rows = rng.integers(0, x_rows * top_k, count)
    rows[[0, 299, 300, 1023]] = x_rows * top_k - 1, x_rows * top_k, -1, 3 * (x_rows // 2)  # X's last row, one that it has not, none
    source = torch.from_numpy(rows // top_k).cuda()
    there = (source >= 0) & (source < x_rows)
    x = exact(X[source.clamp(0, x_rows - 1)] * there.unsqueeze(1))
    offsets = np.concatenate([[0], np.cumsum(sizes)])
    W = values(gen, (E, N, K), "bfloat16")
    ref, terms, _ = go.gemm(x, exact(W), offsets)
    compare(grouped.gemm(X, W, ints(offsets), rows=ints(rows), top_k=top_k), ref, tolerance(X.dtype, ref, terms, K), "product")
    Wt = W.transpose(1, 2).contiguous()
    compare(grouped.gemm(X, Wt, ints(offsets), rows=ints(rows), top_k=top_k, transposed=True), ref, tolerance(X.dtype, ref, terms, K), "transposed")
    dY = values(gen, (count, N), "bfloat16")
    ref, terms, n = go.gemm_grad(dY.double().cpu().numpy(), x, offsets)
    dW = grouped.gemm_grad(dY, X, ints(offsets), rows=ints(rows), top_k=top_k, dtype=torch.float32)
    compare(dW, ref, tolerance(torch.float32, ref, terms, n[:, None, None]), "gradient")

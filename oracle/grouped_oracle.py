"""Plain 64-bit oracle of the products of rows in groups and of the low-rank adapters (numpy, one row after the other where that is clearer)."""
import numpy as np


def sort(ids, E):
    """(offsets, order, place) by lists."""
    flat = np.asarray(ids).reshape(-1).tolist()
    groups = [[] for _ in range(E + 1)]
    for pair, e in enumerate(flat):
        groups[e if 0 <= e < E else E].append(pair)
    order = [p for g in groups for p in g]
    offsets = np.concatenate([[0], np.cumsum([len(g) for g in groups[:E]])])
    place = np.empty(len(flat), np.int64)
    place[np.asarray(order, np.int64)] = np.arange(len(flat))
    return offsets, np.asarray(order, np.int64), place


def source_rows(X, count, rows, top_k):
    """x_i for every i, zeros for a row that X has not."""
    if rows is None:
        return X[:count]
    x = np.zeros((count, X.shape[1]))
    for i, r in enumerate(np.asarray(rows).tolist()):
        if r >= 0 and r // top_k < X.shape[0]:
            x[i] = X[r // top_k]
    return x


def gemm(X, W, offsets, rows=None, top_k=1, transposed=False):
    """(Y, the sums of its terms' magnitudes, whether a group has the row)."""
    count = X.shape[0] if rows is None else len(rows)
    x = source_rows(X, count, rows, top_k)
    N = W.shape[2] if transposed else W.shape[1]
    Y, terms, had = np.zeros((count, N)), np.zeros((count, N)), np.zeros(count, bool)
    for e in range(W.shape[0]):
        at = slice(offsets[e], offsets[e + 1])
        w = W[e] if transposed else W[e].T
        Y[at], terms[at], had[at] = x[at] @ w, np.abs(x[at]) @ np.abs(w), True
    return Y, terms, had


def gemm_grad(dY, X, offsets, rows=None, top_k=1):
    """(dW, the sums of its terms' magnitudes, rows of each group)."""
    x = source_rows(X, dY.shape[0], rows, top_k)
    E = len(offsets) - 1
    dW, terms = np.zeros((E, dY.shape[1], X.shape[1])), np.zeros((E, dY.shape[1], X.shape[1]))
    for e in range(E):
        at = slice(offsets[e], offsets[e + 1])
        dW[e], terms[e] = dY[at].T @ x[at], np.abs(dY[at]).T @ np.abs(x[at])
    return dW, terms, np.diff(offsets)


def lora_add(Y, X, A, B, ids, scaling):
    out = np.array(Y)
    for i, a in enumerate(ids):
        if 0 <= a < len(A):
            out[i] += scaling[a] * (B[a] @ (A[a] @ X[i]))
    return out


def lora_grad(dY, X, A, B, ids, scaling, dX):
    dX, dA, dB = np.array(dX), np.zeros(A.shape), np.zeros(B.shape)
    for i, a in enumerate(ids):
        if 0 <= a < len(A):
            g, h = scaling[a] * (dY[i] @ B[a]), scaling[a] * (A[a] @ X[i])
            dX[i] += g @ A[a]
            dA[a] += np.outer(g, X[i])
            dB[a] += np.outer(dY[i], h)
    return dX, dA, dB

"""Products of rows in groups: experts on 16-bit weights, and their gradients.  ctypes binding of the w4a16_grouped_* functions of
include/w4a16_grouped.h; argument marshalling only, as in `binding`.

    ids, weights = moe.route(logits, top_k)                          # [T, top_k]
    offsets, order, place = grouped.sort(ids, E)
    Y = grouped.gemm(X, W, offsets, rows=order, top_k=top_k)         # X [T, K], W [E, N, K] -> Y [T top_k, N], by expert
    y_tj = Y[place[t, j]]                                            # a token's rows again

    dY -> dX = grouped.gemm(dY, W, offsets, transposed=True)         # [T top_k, K], by expert; a token's gradient is the sum of its rows
    dW = grouped.gemm_grad(dY, X, offsets, rows=order, top_k=top_k)  # [E, N, K]

A call goes to the current stream, or to `stream`; new results come from torch's allocator on the current one.  With another `stream` bring `out` too, or keep the results until it is done.
"""
from __future__ import annotations

import ctypes

from . import mx
from .binding import W4A16Error, _stream

EXPORTS = ("w4a16_grouped_sort_workspace_bytes", "w4a16_grouped_sort", "w4a16_grouped_gemm", "w4a16_grouped_gemm_grad", "w4a16_grouped_query_tile")

_lib = None


def lib():
    """The loaded library with this module's functions declared."""
    global _lib
    if _lib is None:
        L = mx.lib()
        vp, ci, ll, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_longlong, ctypes.c_size_t
        L.w4a16_grouped_sort_workspace_bytes.argtypes = [ll, ci]
        L.w4a16_grouped_sort_workspace_bytes.restype = sz
        L.w4a16_grouped_sort.argtypes = [vp, ll, ci, vp, vp, vp, vp, sz, vp]
        L.w4a16_grouped_gemm.argtypes = [vp, ci, ll, ll, vp, ci, vp, ll, ll, ci, vp, ci, ll, ci, ci, vp, ll, ci, vp]
        L.w4a16_grouped_gemm_grad.argtypes = [vp, ci, ll, vp, ll, ll, vp, ci, vp, ci, ll, ci, ci, vp, ci, ci, vp]
        ip = ctypes.POINTER(ci)
        L.w4a16_grouped_query_tile.argtypes = [ci, ll, ci, ci, ci, ci, ip, ip]
        _lib = L
    return _lib


def _check(rc: int, where: str) -> None:
    if rc:
        raise W4A16Error(rc, where)


def same_device(first, *others) -> None:
    """All on the current device, whose stream the call goes to."""
    import torch
    device = first.device
    if device.type == "cuda" and device.index != torch.cuda.current_device():
        raise ValueError("the tensors are on %s, the current device is cuda:%d" % (device, torch.cuda.current_device()))
    for t in others:
        if t is not None and t.device != device:
            raise ValueError("tensors on %s and %s" % (device, t.device))


def check_ints(t, name: str) -> None:
    import torch
    if not (t.is_cuda and t.dtype is torch.int32 and t.is_contiguous()):
        raise TypeError("%s must be a contiguous CUDA tensor of dtype torch.int32" % name)


def too_large(name: str, shape) -> ValueError:
    """For sizes that the library's 32-bit arguments do not hold; it refuses by itself what is smaller and still too large."""
    return ValueError("%s %r has a size past 32 bits" % (name, tuple(shape)))


def matrix(X, name: str, like=None):
    """(rows, width, leading dimension) of a matrix whose rows are contiguous and 16-byte aligned; `like`: of the same type."""
    if not X.is_cuda or (like is not None and X.dtype is not like.dtype):
        raise TypeError("%s must be a CUDA tensor%s" % (name, "" if like is None else " of dtype %s" % like.dtype))
    if X.dim() != 2:
        raise ValueError("%s must be a matrix, not %r" % (name, tuple(X.shape)))
    found = rows, width, _ = mx.rows_of(X, name)
    if (rows | width) >> 31:
        raise too_large(name, X.shape)
    return found


def query_tile(E: int, count: int, N: int, K: int, transposed: bool = False, grad: bool = False) -> tuple:
    """(rows of a group, columns) of the tiles that gemm, or with `grad` gemm_grad (rows and columns of dW), takes for these sizes; where it is (256, 256), (128, 128) for rows
    gathered from an X of 2 GiB or more."""
    rows, cols = ctypes.c_int(), ctypes.c_int()
    _check(lib().w4a16_grouped_query_tile(E, count, N, K, int(transposed), int(grad), ctypes.byref(rows), ctypes.byref(cols)), "w4a16_grouped_query_tile")
    return rows.value, cols.value


def sort_workspace_bytes(count: int, E: int) -> int:
    """Bytes of workspace that `sort` needs for so many ids; 0 up to 4096."""
    return int(lib().w4a16_grouped_sort_workspace_bytes(count, E))


def sort(ids, E: int, out=None, workspace=None, stream=None):
    """ids int32 (any shape; 0 .. E - 1, anything else: no group) -> (offsets [E + 1], order [count], place [count]), all int32: group e has the places
    offsets[e] .. offsets[e + 1] - 1, order lists the ids' flat numbers by group, in their order inside one and those without a group last, and place
    is its inverse.  `out`: the three to fill, none of them ids.  `workspace`: as in moe.experts, where sort_workspace_bytes is not 0."""
    import torch
    check_ints(ids, "ids")
    count = ids.numel()
    if not 1 <= E <= 1024:
        raise ValueError("1 <= E <= 1024 wanted, not %d" % E)
    if out is None:
        offsets, order, place = (ids.new_empty(n) for n in (E + 1, count, count))
    else:
        offsets, order, place = out
        for t, n, name in ((offsets, E + 1, "offsets"), (order, count, "order"), (place, count, "place")):
            check_ints(t, name)
            if t.numel() != n:
                raise ValueError("%s must have %d values, not %d" % (name, n, t.numel()))
    same_device(ids, offsets, order, place, workspace)
    need = sort_workspace_bytes(count, E)
    if need:
        workspace = brought(workspace, need, ids, stream)
    rc = lib().w4a16_grouped_sort(ids.data_ptr(), count, E, offsets.data_ptr(), order.data_ptr(), place.data_ptr(), workspace.data_ptr() if need else None,
                                  workspace.numel() * workspace.element_size() if need else 0, _stream(stream))
    _check(rc, "w4a16_grouped_sort")
    return offsets, order, place


def brought(workspace, need: int, like, stream):
    """The caller's workspace, checked, or one from torch's allocator on the current stream."""
    import torch
    if workspace is None:
        if stream is not None:
            raise ValueError("with an explicit stream the workspace has to be brought too")
        return torch.empty(need, dtype=torch.uint8, device=like.device)
    if not (workspace.is_cuda and workspace.is_contiguous()):
        raise TypeError("workspace must be a contiguous CUDA tensor")
    return workspace


def _rows(rows, top_k: int, count):
    if rows is None:
        if top_k != 1:
            raise ValueError("top_k goes with rows")
        return
    check_ints(rows, "rows")
    if top_k >> 31 > 0:
        raise too_large("top_k", (top_k,))
    if top_k < 1 or (count is not None and rows.numel() != count):
        raise ValueError("rows must have %s values, top_k be at least 1" % count)


def _offsets(offsets, E: int):
    check_ints(offsets, "offsets")
    if offsets.numel() != E + 1:
        raise ValueError("offsets must have %d values for %d groups, not %d" % (E + 1, E, offsets.numel()))


def gemm(X, W, offsets, rows=None, top_k: int = 1, transposed: bool = False, out=None, stream=None):
    """Y [count, N], Y[i] = W_e x_i for offsets[e] <= i < offsets[e + 1]; x_i = X[i], or X[rows[i] // top_k] with `rows` (sort's order; X [T, K]).
    X float16 or bfloat16 [., K] (a row stride is allowed), W of the same type [E, N, K] or, `transposed`, [E, K, N] (Y[i] = x_i W_e); W may be a view
    whose rows are contiguous.  K and N multiples of 8.  Rows of Y that no group has are 0 in a new Y and stay as they are in `out`, which
    may have a row stride and may not overlap X or W."""
    code = mx.type_code(X.dtype, False)
    x_rows, K, ldx = matrix(X, "X")
    if W.dim() != 3 or not W.is_cuda or W.dtype is not X.dtype:
        raise TypeError("W must be a CUDA tensor [E, %s] of dtype %s" % ("K, N" if transposed else "N, K", X.dtype))
    E, w_rows, w_width = W.shape
    if (E | w_rows | w_width) >> 31:
        raise too_large("W", W.shape)
    N = w_width if transposed else w_rows
    if (w_rows if transposed else w_width) != K:
        raise ValueError("X %r does not fit W %r%s" % (tuple(X.shape), tuple(W.shape), ", transposed" if transposed else ""))
    if w_width > 1 and W.stride(2) != 1:
        raise TypeError("W's rows must be contiguous")
    _offsets(offsets, E)
    _rows(rows, top_k, None)
    count = x_rows if rows is None else rows.numel()
    same_device(X, W, offsets, rows, out)
    Y, ldy = mx._out_matrix(out, count, N, X, X.dtype)
    rc = lib().w4a16_grouped_gemm(X.data_ptr(), code, x_rows, ldx, None if rows is None else rows.data_ptr(), top_k, W.data_ptr(), W.stride(0), W.stride(1),
                                  int(transposed), offsets.data_ptr(), E, count, N, K, Y.data_ptr(), ldy, int(out is None), _stream(stream))
    _check(rc, "w4a16_grouped_gemm")
    return Y


def gemm_grad(dY, X, offsets, rows=None, top_k: int = 1, dtype=None, out=None, accumulate: bool = False, stream=None):
    """dW [E, N, K], dW_e = the sum over the group's rows i of dY[i]^T x_i, x_i as in gemm; zeros for a group without rows.  dY [count, N] and X of the same
    type; dW of `dtype` (X's by default, or float32, or out's type).  `accumulate`: added to what `out` holds
    (contiguous, and apart from dY and X)."""
    import torch
    code = mx.type_code(X.dtype, False)
    x_rows, K, ldx = matrix(X, "X")
    count, N, ldy = matrix(dY, "dY", X)
    check_ints(offsets, "offsets")
    E = offsets.numel() - 1
    _rows(rows, top_k, count)
    if rows is None and x_rows != count:
        raise ValueError("dY %r does not fit X %r" % (tuple(dY.shape), tuple(X.shape)))
    dtype = dtype or (X.dtype if out is None else out.dtype)
    if dtype is not X.dtype and dtype is not torch.float32:
        raise TypeError("gradients in %s or float32, not %s" % (X.dtype, dtype))
    if out is None:
        if accumulate:
            raise ValueError("accumulate goes with out")
        out = torch.empty((E, N, K), dtype=dtype, device=X.device)
    elif not (out.is_cuda and out.is_contiguous() and out.dtype is dtype and tuple(out.shape) == (E, N, K)):
        raise ValueError("out must be a contiguous CUDA tensor [%d, %d, %d] of dtype %s" % (E, N, K, dtype))
    same_device(X, dY, offsets, rows, out)
    rc = lib().w4a16_grouped_gemm_grad(dY.data_ptr(), code, ldy, X.data_ptr(), x_rows, ldx, None if rows is None else rows.data_ptr(), top_k, offsets.data_ptr(), E,
                                       count, N, K, out.data_ptr(), mx.type_code(dtype, True), int(accumulate), _stream(stream))
    _check(rc, "w4a16_grouped_gemm_grad")
    return out

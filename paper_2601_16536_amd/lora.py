"""Low-rank adapters of many requests beside a shared projection, and their gradients.  ctypes binding of the w4a16_lora_* functions of
include/w4a16_grouped.h; argument marshalling only, as in `binding`.

    Y = mx.gemm(X, codes, scales)                       # the projection that all requests share, or binding.gemm
    Y = lora.add(Y, X, A, B, ids, scaling, out=Y)       # + s_a (x A_a^T) B_a^T for the rows of adapter a = ids[row]

    dX, dA, dB = lora.grad(dY, X, A, B, ids, scaling, dX=dX)   # dX: what the shared projection passed back

A [L, R, K] and B [L, N, R] hold L adapters of rank R (a multiple of 8, at most 128; shorter ones end in rows of A and columns of B of zeros), ids int32 [M]
names each row's; a row whose id is outside of 0 .. L - 1 has none.  Streams: as in `grouped`.

The gradient of a shared projection's rows is not this library's: its projections on 4-bit weights have no transposed form, so `dX` comes from the caller (grouped.gemm with `transposed` gives it
for 16-bit weights).
"""
from __future__ import annotations

import ctypes

from . import grouped, mx
from .binding import W4A16Error, _stream

EXPORTS = ("w4a16_lora_workspace_bytes", "w4a16_lora_add", "w4a16_lora_grad")

_lib = None


def lib():
    """The loaded library with this module's functions declared."""
    global _lib
    if _lib is None:
        L = mx.lib()
        vp, ci, ll, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_longlong, ctypes.c_size_t
        L.w4a16_lora_workspace_bytes.argtypes = [ci] * 6
        L.w4a16_lora_workspace_bytes.restype = sz
        L.w4a16_lora_add.argtypes = [vp, ll, vp, ci, ll, vp, vp, vp, vp, ci, ci, ci, ci, ci, vp, ll, vp, sz, vp]
        L.w4a16_lora_grad.argtypes = [vp, ll, vp, ci, ll, vp, vp, vp, vp, ci, ci, ci, ci, ci, vp, ll, vp, ll, vp, vp, ci, vp, sz, vp]
        _lib = L
    return _lib


def workspace_bytes(M: int, L: int, R: int, K: int, N: int, grad: bool = False) -> int:
    """Bytes of workspace that `add`, or with `grad` `grad`, needs."""
    return int(lib().w4a16_lora_workspace_bytes(M, L, R, K, N, int(grad)))


def _check(X, A, B, ids, scaling, other, name: str):
    """(type, M, L, R, K, N, X's leading dimension, other's) of a call; `other`: the matrix [M, N] beside X."""
    import torch
    code = mx.type_code(X.dtype, False)
    M, K, ldx = grouped.matrix(X, "X")
    M2, N, ld = grouped.matrix(other, name, X)
    for t, n in ((A, "A"), (B, "B")):
        if not (t.is_cuda and t.dtype is X.dtype and t.is_contiguous() and t.dim() == 3):
            raise TypeError("%s must be a contiguous CUDA tensor of three dimensions and dtype %s" % (n, X.dtype))
    L, R, _ = A.shape
    if M2 != M or A.shape[2] != K or tuple(B.shape) != (L, N, R):
        raise ValueError("X %r, %s %r, A %r and B %r do not fit each other" % (tuple(X.shape), name, tuple(other.shape), tuple(A.shape), tuple(B.shape)))
    if (L | R) >> 31:
        raise grouped.too_large("A", A.shape)
    grouped.check_ints(ids, "ids")
    if ids.numel() != M:
        raise ValueError("ids must have %d values, not %d" % (M, ids.numel()))
    if scaling is not None:
        if not (scaling.is_cuda and scaling.dtype is torch.float32 and scaling.is_contiguous()):
            raise TypeError("scaling must be a contiguous CUDA tensor of dtype torch.float32")
        if scaling.numel() != L:
            raise ValueError("scaling must have %d values, not %d" % (L, scaling.numel()))
    return code, M, L, R, K, N, ldx, ld


def add(Y, X, A, B, ids, scaling=None, out=None, workspace=None, stream=None):
    """Y + scaling[a] (x A_a^T) B_a^T, a = ids[row], [M, N]; rows without an adapter as they are.  Y, X [M, K], A and B float16 or all bfloat16, Y and X with a row
    stride if need be; scaling float32 [L] (by default 1).  The result is a new tensor, or `out`, which may be Y itself and may not overlap X.  `workspace`: as in moe.experts,
    of workspace_bytes(M, L, R, K, N)."""
    code, M, L, R, K, N, ldx, ldy = _check(X, A, B, ids, scaling, Y, "Y")
    out, ldo = mx._out_matrix(out, M, N, X, X.dtype)
    grouped.same_device(X, Y, A, B, ids, scaling, out, workspace)
    workspace = grouped.brought(workspace, workspace_bytes(M, L, R, K, N), X, stream)
    rc = lib().w4a16_lora_add(Y.data_ptr(), ldy, X.data_ptr(), code, ldx, A.data_ptr(), B.data_ptr(), ids.data_ptr(), None if scaling is None else scaling.data_ptr(),
                              M, L, R, K, N, out.data_ptr(), ldo, workspace.data_ptr(), workspace.numel() * workspace.element_size(), _stream(stream))
    if rc:
        raise W4A16Error(rc, "w4a16_lora_add")
    return out


def grad(dY, X, A, B, ids, scaling=None, dX=None, dtype=None, out=None, workspace=None, stream=None):
    """(dX + scaling[a] (dy B_a) A_a, dA [L, R, K], dB [L, N, R]) for add's arguments and the gradient dY [M, N] of its result.  dX [M, K]: what the shared
    projection passed back (by default 0).  dA and dB of `dtype`: X's by default, or float32; zeros for an adapter without rows.  `out`: the three to fill, the first
    of which may be dX itself; none may overlap dY, X, A or B.  `workspace`: of workspace_bytes(M, L, R, K, N, grad=True)."""
    import torch
    code, M, L, R, K, N, ldx, ldy = _check(X, A, B, ids, scaling, dY, "dY")
    lddx = 0
    if dX is not None:
        if tuple(dX.shape) != (M, K):
            raise ValueError("dX must be [%d, %d], not %r" % (M, K, tuple(dX.shape)))
        _, _, lddx = grouped.matrix(dX, "dX", X)
    if out is None:
        dtype = dtype or X.dtype
        to, dA, dB = None, torch.empty(A.shape, dtype=dtype, device=X.device), torch.empty(B.shape, dtype=dtype, device=X.device)
    else:
        to, dA, dB = out
        dtype = dtype or dA.dtype
        for t, like, name in ((dA, A, "dA"), (dB, B, "dB")):
            if not (t.is_cuda and t.is_contiguous() and t.dtype is dtype and t.shape == like.shape):
                raise ValueError("%s must be a contiguous CUDA tensor %r of dtype %s" % (name, tuple(like.shape), dtype))
    if dtype is not X.dtype and dtype is not torch.float32:
        raise TypeError("gradients in %s or float32, not %s" % (X.dtype, dtype))
    to, ldo = mx._out_matrix(to, M, K, X, X.dtype)
    grouped.same_device(X, dY, A, B, ids, scaling, dX, to, dA, dB, workspace)
    workspace = grouped.brought(workspace, workspace_bytes(M, L, R, K, N, True), X, stream)
    rc = lib().w4a16_lora_grad(dY.data_ptr(), ldy, X.data_ptr(), code, ldx, A.data_ptr(), B.data_ptr(), ids.data_ptr(), None if scaling is None else scaling.data_ptr(),
                               M, L, R, K, N, None if dX is None else dX.data_ptr(), lddx, to.data_ptr(), ldo, dA.data_ptr(), dB.data_ptr(),
                               mx.type_code(dtype, True), workspace.data_ptr(), workspace.numel() * workspace.element_size(), _stream(stream))
    if rc:
        raise W4A16Error(rc, "w4a16_lora_grad")
    return to, dA, dB

"""Microscaled 4-bit floating point (MXFP4): quantisation, read-back and products.  ctypes binding of the w4a16_mx_*
functions of include/w4a16_mx.h; argument marshalling only, as in `binding`.

A matrix [..., rows, K] in MXFP4 is two tensors: codes uint8 [..., rows, K/2] (the even k in the low nibble) and scales
uint8 [..., rows, K/32].  K is a multiple of 32.

    codes, scales = mx.quantize(W)            # W [N, K], fp16, bf16 or fp32
    Y = mx.gemm(X, codes, scales)             # X [M, K] fp16 or bf16 -> Y [M, N] = X W^T
    xc, xs = mx.quantize(X)
    Y = mx.gemm_mx(xc, xs, codes, scales)     # both operands in four bits
"""
from __future__ import annotations

import ctypes

from . import binding
from .binding import W4A16Error, _stream

F16, BF16, F32 = 0, 1, 2

EXPORTS = ("w4a16_mx_quantize", "w4a16_mx_dequantize", "w4a16_mx_gemm", "w4a16_mx_gemm_mx", "w4a16_mx_query_tile", "w4a16_mx_query_lds")

_lib = None
_types = None
_u8 = None


def lib():
    """The loaded library with this module's functions declared."""
    global _lib, _types, _u8
    if _lib is None:
        import torch
        L = binding.lib()
        vp, ci, ll = ctypes.c_void_p, ctypes.c_int, ctypes.c_longlong
        L.w4a16_mx_quantize.argtypes = [vp, ci, ll, ci, ll, vp, vp, vp]
        L.w4a16_mx_dequantize.argtypes = [vp, vp, ll, ci, vp, ci, ll, vp]
        L.w4a16_mx_gemm.argtypes = [vp, ci, ll, vp, vp, ci, ci, ci, vp, ll, vp]
        L.w4a16_mx_gemm_mx.argtypes = [vp, vp, vp, vp, ci, ci, ci, vp, ci, ll, vp]
        ip = ctypes.POINTER(ci)
        L.w4a16_mx_query_tile.argtypes = [ci, ci, ci, ci, ci, ip, ip]
        L.w4a16_mx_query_lds.argtypes = L.w4a16_mx_query_tile.argtypes
        _types = {torch.float16: F16, torch.bfloat16: BF16, torch.float32: F32}
        _u8 = torch.uint8
        _lib = L
    return _lib


def _check(rc: int, where: str) -> None:
    if rc:
        raise W4A16Error(rc, where)


def type_code(dtype, wide: bool) -> int:
    """The library's number of a torch dtype; `wide`: float32 is allowed too."""
    if _lib is None:
        lib()
    code = _types.get(dtype)
    if code is None or (code == F32 and not wide):
        raise TypeError("float16%s or bfloat16 wanted, not %s" % (", float32" if wide else "", dtype))
    return code


def rows_of(X, name: str):
    """(rows, K, leading dimension) of a matrix, or of a contiguous tensor seen as one."""
    if not X.is_cuda:
        raise TypeError("%s must be a CUDA tensor" % name)
    if X.dim() == 2 and (X.stride(1) == 1 or X.shape[1] == 1):
        rows, K = X.shape
        return rows, K, (X.stride(0) if rows > 1 else K)
    if X.dim() < 1 or not X.is_contiguous():
        raise TypeError("%s must be a matrix whose rows are contiguous, or a contiguous tensor" % name)
    K = X.shape[-1]
    return (X.numel() // K if K else 0), K, K


def check_mx(codes, scales, name: str):
    """(leading shape, K) of an MXFP4 pair of tensors."""
    if _u8 is None:
        lib()
    if not (codes.dtype is _u8 and scales.dtype is _u8 and codes.is_cuda and scales.is_cuda and codes.is_contiguous() and scales.is_contiguous()):
        raise TypeError("%s: codes and scales must be contiguous CUDA tensors of dtype torch.uint8" % name)
    cs, ss = codes.shape, scales.shape
    lead = cs[:-1]
    if lead != ss[:-1] or not cs[-1] or cs[-1] != 16 * ss[-1]:
        raise ValueError("%s: codes %r and scales %r do not fit each other (K / 2 and K / 32 to a row)" % (name, tuple(cs), tuple(ss)))
    return lead, 2 * cs[-1]


def _out_matrix(out, M: int, N: int, like, dtype):
    """The output [M, N] and its leading dimension: new, or `out` checked."""
    if out is None:
        return (like.new_empty((M, N)) if like.dtype is dtype else like.new_empty((M, N), dtype=dtype)), N
    if not out.is_cuda or out.dtype is not dtype or tuple(out.shape) != (M, N) or (N > 1 and out.stride(1) != 1) or (M > 1 and out.stride(0) < N):
        raise ValueError("out must be a CUDA tensor [%d, %d] of dtype %s whose rows are contiguous" % (M, N, dtype))
    return out, (out.stride(0) if M > 1 else N)


def query_tile(M: int, N: int, K: int, dtype=None, x_mx: bool = False) -> tuple:
    """(rows of X, columns of Y) that a workgroup of gemm (dtype: X's), or with x_mx of gemm_mx, takes for this shape; 16 columns: the kernel for few rows."""
    import torch
    tm, tn = ctypes.c_int(), ctypes.c_int()
    _check(lib().w4a16_mx_query_tile(M, N, K, type_code(dtype or torch.bfloat16, False), int(x_mx), ctypes.byref(tm), ctypes.byref(tn)), "w4a16_mx_query_tile")
    return tm.value, tn.value


def query_lds(M: int, N: int, K: int, dtype=None, x_mx: bool = False) -> tuple:
    """(bytes of LDS of a workgroup of that kernel, pieces of K that X passes through it in)."""
    import torch
    lds, chunks = ctypes.c_int(), ctypes.c_int()
    _check(lib().w4a16_mx_query_lds(M, N, K, type_code(dtype or torch.bfloat16, False), int(x_mx), ctypes.byref(lds), ctypes.byref(chunks)), "w4a16_mx_query_lds")
    return lds.value, chunks.value


def quantize(X, out=None, stream=None):
    """X [..., K] -> (codes uint8 [..., K/2], scales uint8 [..., K/32]).  A matrix may have a row stride.  `out`: the pair to fill."""
    code = type_code(X.dtype, True)
    rows, K, ld = rows_of(X, "X")
    if K < 32 or K % 32:
        raise ValueError("the last dimension must be a multiple of 32, not %d" % K)
    lead = X.shape[:-1]
    if out is None:
        codes = X.new_empty((*lead, K // 2), dtype=_u8)
        scales = X.new_empty((*lead, K // 32), dtype=_u8)
    else:
        codes, scales = out
        if check_mx(codes, scales, "out") != (lead, K):
            raise ValueError("out does not fit X %r" % (tuple(X.shape),))
    _check(lib().w4a16_mx_quantize(X.data_ptr(), code, rows, K, ld, codes.data_ptr(), scales.data_ptr(), _stream(stream)), "w4a16_mx_quantize")
    return codes, scales


def dequantize(codes, scales, dtype=None, out=None, stream=None):
    """The matrix that codes and scales stand for, in float16, bfloat16 (the default) or float32; `out` may have a row stride."""
    import torch
    lead, K = check_mx(codes, scales, "dequantize")
    if out is None:
        out = torch.empty((*lead, K), dtype=dtype or torch.bfloat16, device=codes.device)
    elif tuple(out.shape) != (*lead, K) or (dtype is not None and out.dtype is not dtype):
        raise ValueError("out must have shape %r%s" % ((*lead, K), "" if dtype is None else " and dtype %s" % dtype))
    code = type_code(out.dtype, True)
    rows, _, ld = rows_of(out, "out")
    _check(lib().w4a16_mx_dequantize(codes.data_ptr(), scales.data_ptr(), rows, K, out.data_ptr(), code, ld, _stream(stream)), "w4a16_mx_dequantize")
    return out


def gemm(X, codes, scales, out=None, stream=None):
    """Y [M, N] = X W^T with X [M, K] in float16 or bfloat16 (rows 16-byte aligned; a row stride is allowed) and W [N, K] in MXFP4."""
    code = type_code(X.dtype, False)
    lead, K = check_mx(codes, scales, "W")
    M, KX, ld = rows_of(X, "X")
    if X.dim() != 2 or len(lead) != 1 or KX != K:
        raise ValueError("X %r does not fit W [%s, %d]" % (tuple(X.shape), ", ".join(map(str, lead)), K))
    N = lead[0]
    Y, ldy = _out_matrix(out, M, N, X, X.dtype)
    rc = lib().w4a16_mx_gemm(X.data_ptr(), code, ld, codes.data_ptr(), scales.data_ptr(), M, N, K, Y.data_ptr(), ldy, _stream(stream))
    _check(rc, "w4a16_mx_gemm")
    return Y


def gemm_mx(x_codes, x_scales, codes, scales, dtype=None, out=None, stream=None):
    """Y [M, N] = X W^T with X [M, K] and W [N, K] both in MXFP4; Y in float16 or bfloat16 (the default, or out's type)."""
    import torch
    if dtype is None:
        dtype = torch.bfloat16 if out is None else out.dtype
    code = type_code(dtype, False)
    lead, K = check_mx(codes, scales, "W")
    lead_x, KX = check_mx(x_codes, x_scales, "X")
    if len(lead) != 1 or len(lead_x) != 1 or KX != K:
        raise ValueError("X [%s, %d] does not fit W [%s, %d]" % (", ".join(map(str, lead_x)), KX, ", ".join(map(str, lead)), K))
    M, N = lead_x[0], lead[0]
    Y, ldy = _out_matrix(out, M, N, codes, dtype)
    rc = lib().w4a16_mx_gemm_mx(x_codes.data_ptr(), x_scales.data_ptr(), codes.data_ptr(), scales.data_ptr(), M, N, K, Y.data_ptr(), code, ldy,
                                _stream(stream))
    _check(rc, "w4a16_mx_gemm_mx")
    return Y

"""A mixture-of-experts layer on MXFP4 weights: the router's choice and the experts' feed-forward layers.  ctypes binding of the
w4a16_moe_* functions of include/w4a16_mx.h; argument marshalling only, as in `binding`.

    w13, s13 = mx.quantize(W13)     # W13 [E, 2 I, H]: each expert's gate rows, then its up rows
    w2, s2 = mx.quantize(W2)        # W2 [E, H, I]
    ids, weights = moe.route(logits, top_k)
    Y = moe.experts(X, ids, weights, w13, s13, w2, s2)
"""
from __future__ import annotations

import ctypes

from . import mx
from .binding import W4A16Error, _stream

SCORINGS = {"softmax": 0, "sigmoid": 1}
ACTIVATIONS = {"silu": 0, "gelu": 1}

EXPORTS = ("w4a16_moe_route", "w4a16_moe_workspace_bytes", "w4a16_moe_experts", "w4a16_moe_query_plan")

_lib = None


class Plan(ctypes.Structure):
    _fields_ = [(name, ctypes.c_int) for name in ("tiles", "rows_up", "rows_down", "lds_up", "lds_down")]


def lib():
    """The loaded library with this module's functions declared."""
    global _lib
    if _lib is None:
        L = mx.lib()
        vp, ci, ll, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_longlong, ctypes.c_size_t
        L.w4a16_moe_route.argtypes = [vp, ci, ci, ci, ll, ci, ci, ci, ctypes.c_float, vp, vp, vp]
        L.w4a16_moe_workspace_bytes.argtypes = [ci, ci, ci, ci]
        L.w4a16_moe_workspace_bytes.restype = sz
        L.w4a16_moe_experts.argtypes = [vp, ci, ll, vp, vp, vp, vp, vp, vp, ci, ci, ci, ci, ci, ci, vp, ll, vp, sz, vp]
        L.w4a16_moe_query_plan.argtypes = [ci, ci, ci, ci, ci, ctypes.POINTER(Plan)]
        _lib = L
    return _lib


def workspace_bytes(T: int, top_k: int, H: int, I: int) -> int:
    """Bytes of workspace that `experts` needs."""
    return int(lib().w4a16_moe_workspace_bytes(T, top_k, H, I))


def query_plan(T: int, E: int, top_k: int, H: int, I: int) -> dict:
    """What `experts` runs for a layer of these sizes: `tiles` or streamed weights; rows of an expert at a time and bytes of LDS of a workgroup of the gate and up
    product and of the down product."""
    p = Plan()
    rc = lib().w4a16_moe_query_plan(T, E, top_k, H, I, ctypes.byref(p))
    if rc:
        raise W4A16Error(rc, "w4a16_moe_query_plan")
    return {name: getattr(p, name) for name, _ in Plan._fields_}


def route(logits, top_k: int, scoring: str = "softmax", renormalize: bool = True, factor: float = 1.0, out=None, stream=None):
    """logits [T, E] (float16, bfloat16 or float32; a row stride is allowed) -> (ids int32 [T, top_k], weights float32 [T, top_k]):
    the experts of the largest logits, in descending order, ties to the lowest index.  A logit of -inf excludes its expert
    (id -1, weight 0 where none is left).  `out`: the pair to fill."""
    import torch
    code = mx.type_code(logits.dtype, True)
    if logits.dim() != 2 or scoring not in SCORINGS:
        raise ValueError("logits [T, E] and scoring 'softmax' or 'sigmoid' wanted")
    T, E, ld = mx.rows_of(logits, "logits")
    if not 1 <= top_k <= min(E, 32) or E > 1024:
        raise ValueError("1 <= top_k <= 32, top_k <= E <= 1024 wanted, not top_k %d of %d" % (top_k, E))
    if out is None:
        ids = logits.new_empty((T, top_k), dtype=torch.int32)
        weights = logits.new_empty((T, top_k), dtype=torch.float32)
    else:
        ids, weights = out
        _check_choice(ids, weights, T)
        if ids.shape[1] != top_k:
            raise ValueError("out must be a pair [%d, %d]" % (T, top_k))
    rc = lib().w4a16_moe_route(logits.data_ptr(), code, T, E, ld, top_k, SCORINGS[scoring], bool(renormalize), factor, ids.data_ptr(),
                               weights.data_ptr(), _stream(stream))
    if rc:
        raise W4A16Error(rc, "w4a16_moe_route")
    return ids, weights


def _check_choice(ids, weights, T: int) -> None:
    import torch
    if not (ids.is_cuda and weights.is_cuda and ids.dtype is torch.int32 and weights.dtype is torch.float32 and ids.is_contiguous()
            and weights.is_contiguous()):
        raise TypeError("ids must be a contiguous CUDA tensor of dtype torch.int32, weights of torch.float32")
    if ids.dim() != 2 or ids.shape != weights.shape or ids.shape[0] != T:
        raise ValueError("ids %r and weights %r do not fit %d tokens" % (tuple(ids.shape), tuple(weights.shape), T))


def experts(X, ids, weights, codes13, scales13, codes2, scales2, activation: str = "silu", out=None, workspace=None, stream=None):
    """Y [T, H]: for every token the weighted sum of its experts' W2 (act(W1 x) * (W3 x)).  X [T, H] float16 or bfloat16; codes13, scales13
    of [E, 2 I, H], codes2, scales2 of [E, H, I] in MXFP4; activation 'silu' or 'gelu'.  `workspace`: a contiguous CUDA tensor of
    workspace_bytes(T, top_k, H, I), 256-byte aligned, this call's own until its work is done; by default one from torch's allocator
    (on the current stream: with an explicit stream bring one)."""
    import torch
    code = mx.type_code(X.dtype, False)
    lead13, H = mx.check_mx(codes13, scales13, "W13")
    lead2, I = mx.check_mx(codes2, scales2, "W2")
    T, HX, ld = mx.rows_of(X, "X")
    if X.dim() != 2 or len(lead13) != 2 or len(lead2) != 2 or HX != H or lead13[0] != lead2[0] or lead13[1] != 2 * I or lead2[1] != H:
        raise ValueError("X %r, W13 %r and W2 %r do not fit each other" % (tuple(X.shape), (*lead13, H), (*lead2, I)))
    if activation not in ACTIVATIONS:
        raise ValueError("activation must be 'silu' or 'gelu'")
    _check_choice(ids, weights, T)
    top_k = ids.shape[1]
    Y, ldy = mx._out_matrix(out, T, H, X, X.dtype)
    need = T * top_k * (H + I) * 4
    if workspace is None:
        if stream is not None:
            raise ValueError("with an explicit stream the workspace has to be brought too")
        workspace = torch.empty(need, dtype=torch.uint8, device=X.device)
    elif not (workspace.is_cuda and workspace.is_contiguous()):
        raise TypeError("workspace must be a contiguous CUDA tensor")
    rc = lib().w4a16_moe_experts(X.data_ptr(), code, ld, ids.data_ptr(), weights.data_ptr(), codes13.data_ptr(), scales13.data_ptr(), codes2.data_ptr(),
                                 scales2.data_ptr(), T, lead13[0], top_k, H, I, ACTIVATIONS[activation], Y.data_ptr(), ldy, workspace.data_ptr(),
                                 workspace.numel() * workspace.element_size(), _stream(stream))
    if rc:
        raise W4A16Error(rc, "w4a16_moe_experts")
    return Y

"""ctypes binding of include/ffn24_block.h: layer norm, the gated feed-forward block, int8 products.

Like the binding of ffn24.h it only marshals arguments: torch allocates and owns the tensors, every call enqueues on torch's current stream, and
what does not fit is refused with ValueError (shapes, types, contiguity, checked here) or Ffn24Error (checked by the library).
"""
from __future__ import annotations

import ctypes

import torch

from . import ffn24
from .ffn24 import Ffn24Error, _BF16, _F32, _check, _expect, _ptr, _stream  # noqa: F401

EXPORTS = ("layer_norm_fwd", "layer_norm_bwd_scratch", "layer_norm_bwd")

_lib = None


def lib() -> ctypes.CDLL:
    """libffn24.so with the argument types of this half of it."""
    global _lib
    if _lib is None:
        L = ffn24.lib()
        vp, i64, ci, f32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_float
        L.layer_norm_fwd.argtypes = [vp, vp, vp, vp, i64, i64, f32, ci, vp, vp, vp, vp, vp]
        L.layer_norm_bwd_scratch.argtypes = [i64, i64]
        L.layer_norm_bwd.argtypes = [vp, vp, vp, vp, vp, vp, i64, i64, ci, vp, vp, vp, vp, vp]
        for name in EXPORTS:
            getattr(L, name).restype = ci
        L.layer_norm_bwd_scratch.restype = i64
        _lib = L
    return _lib


# ---------------------------------------------------------------------------------------------- layer norm
_NORM_TYPES = {torch.bfloat16: 0, torch.float32: 1}


def layer_norm_fwd(X, weight, bias=None, eps: float = 1e-5, residual=None):
    """Layer norm of the rows of X [T, D] (bf16 or fp32), of X + residual if one is given; weight, bias fp32 [D].

    Returns (Y, S, mean, rstd): S is the sum, rounded to X's type (X itself without a residual), mean and rstd are fp32 [T]; layer_norm_bwd takes the
    last three."""
    T, D = X.shape
    _expect(X, (T, D), _NORM_TYPES, "X")
    _expect(residual, (T, D), (X.dtype,), "residual")
    _expect(weight, (D,), _F32, "weight")
    _expect(bias, (D,), _F32, "bias")
    Y = torch.empty_like(X)
    S = torch.empty_like(X) if residual is not None else None
    stat = torch.empty((2, (T + 3) & ~3), dtype=torch.float32, device=X.device)
    mean, rstd = stat[0, :T], stat[1, :T]
    _check(lib().layer_norm_fwd(_ptr(X), _ptr(residual), _ptr(weight), _ptr(bias), T, D, eps, _NORM_TYPES[X.dtype], _ptr(S), _ptr(Y), _ptr(mean), _ptr(rstd),
                                _stream()), "layer_norm_fwd")
    return Y, X if S is None else S, mean, rstd


def layer_norm_bwd(dY, S, weight, mean, rstd, dS=None):
    """Gradients of layer_norm_fwd: (dX, dweight, dbias); dX is that of X and of the residual, with dS, what reaches S beside the norm, added."""
    T, D = S.shape
    _expect(S, (T, D), _NORM_TYPES, "S")
    _expect(dY, (T, D), (S.dtype,), "dY")
    _expect(dS, (T, D), (S.dtype,), "dS")
    _expect(weight, (D,), _F32, "weight")
    _expect(mean, (T,), _F32, "mean")
    _expect(rstd, (T,), _F32, "rstd")
    dX = torch.empty_like(S)
    dw, db = torch.empty(D, dtype=torch.float32, device=S.device), torch.empty(D, dtype=torch.float32, device=S.device)
    scratch = torch.empty(max(int(lib().layer_norm_bwd_scratch(T, D)), 0), dtype=torch.uint8, device=S.device)
    _check(lib().layer_norm_bwd(_ptr(dY), _ptr(S), _ptr(weight), _ptr(mean), _ptr(rstd), _ptr(dS), T, D, _NORM_TYPES[S.dtype], _ptr(dX), _ptr(dw), _ptr(db),
                                _ptr(scratch), _stream()), "layer_norm_bwd")
    return dX, dw, db

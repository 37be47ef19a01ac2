"""ctypes binding of include/ffn24_block.h: layer norm, the gated feed-forward block, int8 products.

Like the binding of ffn24.h it only marshals arguments: torch allocates and owns the tensors, every call enqueues on torch's current stream, and
what does not fit is refused with ValueError (shapes, types, contiguity, the device, checked here) or Ffn24Error (checked by the library).
"""
from __future__ import annotations

import ctypes

import torch

from . import ffn24
from .ffn24 import Ffn24Error, _BF16, _F32, _check, _expect, _ptr

EXPORTS = ("layer_norm_fwd", "layer_norm_bwd_scratch", "layer_norm_bwd", "gated_ctx_create", "gated_ctx_destroy", "gated_fwd", "gated_bwd",
           "i8_weight_bytes", "i8_weight", "quantise_i8", "matmul_i8", "linear_i8_scratch", "linear_i8", "gated_i8_ctx_create", "gated_i8_ctx_destroy",
           "gated_i8_set_weights", "gated_i8_fwd")

_lib = None


def _stream(*tensors) -> int:
    """torch's current stream, as a number (torch.cuda.current_stream builds an object first: 2.8 us a call, this 0.1).  The library launches on the current device, so all
    tensors of the call have to be there."""
    device = torch._C._cuda_getDevice()
    for t in tensors:
        if t is not None and t.get_device() != device:
            raise ValueError(f"a tensor is on device {t.get_device()}, the current device is {device}")
    return torch._C._cuda_getCurrentRawStream(device)


def lib() -> ctypes.CDLL:
    """libffn24.so with the argument types of this half of it."""
    global _lib
    if _lib is None:
        L = ffn24.lib()
        vp, i64, ci, f32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_float
        L.layer_norm_fwd.argtypes = [vp, vp, vp, vp, i64, i64, f32, ci, vp, vp, vp, vp, vp]
        L.layer_norm_bwd_scratch.argtypes = [i64, i64]
        L.layer_norm_bwd.argtypes = [vp, vp, vp, vp, vp, vp, i64, i64, ci, vp, vp, vp, vp, vp]
        L.gated_ctx_create.argtypes = [ctypes.POINTER(vp), i64, i64, i64, ci, ci]
        L.gated_ctx_destroy.argtypes = [vp]
        L.gated_fwd.argtypes = [vp, vp, i64, vp, vp, vp, vp]
        L.gated_bwd.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp]
        L.i8_weight_bytes.argtypes = [i64, i64]
        L.i8_weight.argtypes = [vp, i64, i64, ci, vp, vp]
        L.quantise_i8.argtypes = [vp, i64, i64, vp, vp, vp]
        L.matmul_i8.argtypes = [vp, vp, i64, vp, i64, i64, vp, vp]
        L.linear_i8_scratch.argtypes = [i64, i64, i64]
        L.linear_i8.argtypes = [vp, i64, vp, i64, i64, vp, vp, vp]
        L.gated_i8_ctx_create.argtypes = [ctypes.POINTER(vp), i64, i64, i64, ci]
        L.gated_i8_ctx_destroy.argtypes = [vp]
        L.gated_i8_set_weights.argtypes = [vp, vp, vp, vp]
        L.gated_i8_fwd.argtypes = [vp, vp, i64, vp, vp]
        for name in EXPORTS:
            getattr(L, name).restype = ci
        L.layer_norm_bwd_scratch.restype = L.i8_weight_bytes.restype = L.linear_i8_scratch.restype = i64
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
    mean, rstd = torch.empty(T, dtype=torch.float32, device=X.device), torch.empty(T, dtype=torch.float32, device=X.device)
    _check(lib().layer_norm_fwd(_ptr(X), _ptr(residual), _ptr(weight), _ptr(bias), T, D, eps, _NORM_TYPES[X.dtype], _ptr(S), _ptr(Y), _ptr(mean), _ptr(rstd),
                                _stream(X, residual, weight, bias)), "layer_norm_fwd")
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
                                _ptr(scratch), _stream(S, dY, dS, weight, mean, rstd)), "layer_norm_bwd")
    return dX, dw, db


# ---------------------------------------------------------------------------------------------- gated feed-forward block
GATES = {"silu": 0, "gelu": 1}


def _gate(act: str) -> int:
    if act not in GATES:
        raise ValueError(f"act: {act!r}, expected one of {tuple(GATES)}")
    return GATES[act]


class _Handle:
    """Owns a context of the library, on the device that was current at its creation; the subclass names its destructor."""
    _h = None
    _destroy = ""

    def _own(self, h):
        self._h, self._device = h, torch.cuda.current_device()

    def close(self):
        if self._h:
            torch.cuda.synchronize(self._device)
            _check(getattr(lib(), self._destroy)(self._h), self._destroy)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class GatedContext(_Handle):
    """The gated feed-forward block (see gated_ctx in the header) for up to T tokens: Y = (a(X Wg) * (X Wu)) Wd with Wgu = [Wg | Wu] [D, 2 F], Wd [F, D],
    all bf16; act "silu" or "gelu" (its tanh form)."""
    _destroy = "gated_ctx_destroy"

    def __init__(self, T: int, D: int, F: int, act: str = "silu", training: bool = False):
        self.T, self.D, self.F, self.training = T, D, F, training
        h = ctypes.c_void_p()
        _check(lib().gated_ctx_create(ctypes.byref(h), T, D, F, _gate(act), ffn24.FFN24_TRAINING if training else 0), "gated_ctx_create")
        self._own(h)

    def _expect_weights(self, Wgu, Wd):
        _expect(Wgu, (self.D, 2 * self.F), _BF16, "Wgu")
        _expect(Wd, (self.F, self.D), _BF16, "Wd")

    def fwd(self, X, Wgu, Wd, Y=None):
        """X [t, D] with any t up to T -> Y [t, D]."""
        t = X.shape[0]
        _expect(X, (t, self.D), _BF16, "X")
        self._expect_weights(Wgu, Wd)
        Y = torch.empty_like(X) if Y is None else Y
        _expect(Y, (t, self.D), _BF16, "Y")
        _check(lib().gated_fwd(self._h, _ptr(X), t, _ptr(Wgu), _ptr(Wd), _ptr(Y), _stream(X, Wgu, Wd, Y)), "gated_fwd")
        self._t = t
        return Y

    def bwd(self, dY, X, Wgu, Wd, out=None):
        """Gradients of the last fwd, which had this X and these weights: (dX, dWgu, dWd)."""
        t = getattr(self, "_t", X.shape[0])
        _expect(dY, (t, self.D), _BF16, "dY")
        _expect(X, (t, self.D), _BF16, "X")
        self._expect_weights(Wgu, Wd)
        dX, dWgu, dWd = (torch.empty_like(X), torch.empty_like(Wgu), torch.empty_like(Wd)) if out is None else out
        _expect(dX, (t, self.D), _BF16, "dX")
        _expect(dWgu, (self.D, 2 * self.F), _BF16, "dWgu")
        _expect(dWd, (self.F, self.D), _BF16, "dWd")
        _check(lib().gated_bwd(self._h, _ptr(dY), _ptr(X), _ptr(Wgu), _ptr(Wd), _ptr(dX), _ptr(dWgu), _ptr(dWd), _stream(dY, X, Wgu, Wd, dX, dWgu, dWd)), "gated_bwd")
        return dX, dWgu, dWd


# ---------------------------------------------------------------------------------------------- 8-bit integer products
_I8 = (torch.int8,)


def _size(nbytes: int, what: str) -> int:
    if nbytes < 0:
        raise Ffn24Error(-2, what)
    return nbytes


class I8Weight:
    """W [K, N] (bf16) quantised per output channel and laid out for linear_i8 and matmul_i8 (see i8_weight in the header); W is not needed afterwards."""

    def __init__(self, W):
        self.K, self.N = W.shape
        _expect(W, (self.K, self.N), _BF16, "W")
        self.data = torch.empty(_size(int(lib().i8_weight_bytes(self.K, self.N)), "i8_weight"), dtype=torch.uint8, device=W.device)
        _check(lib().i8_weight(_ptr(W), self.K, self.N, 0, _ptr(self.data), _stream(W)), "i8_weight")


def quantise_i8(X, codes=None, scales=None):
    """X [T, K] (bf16) -> (codes [T, K] int8, scales [T] fp32): X = codes * scales to within half a scale."""
    T, K = X.shape
    _expect(X, (T, K), _BF16, "X")
    codes = torch.empty((T, K), dtype=torch.int8, device=X.device) if codes is None else codes
    scales = torch.empty((T,), dtype=torch.float32, device=X.device) if scales is None else scales
    _expect(codes, (T, K), _I8, "codes")
    _expect(scales, (T,), _F32, "scales")
    _check(lib().quantise_i8(_ptr(X), T, K, _ptr(codes), _ptr(scales), _stream(X, codes, scales)), "quantise_i8")
    return codes, scales


def matmul_i8(codes, scales, W: I8Weight, Y=None):
    """Y [T, N] (bf16) from the codes and scales of quantise_i8."""
    T = codes.shape[0]
    _expect(codes, (T, W.K), _I8, "codes")
    _expect(scales, (T,), _F32, "scales")
    Y = torch.empty((T, W.N), dtype=torch.bfloat16, device=codes.device) if Y is None else Y
    _expect(Y, (T, W.N), _BF16, "Y")
    _check(lib().matmul_i8(_ptr(codes), _ptr(scales), T, _ptr(W.data), W.K, W.N, _ptr(Y), _stream(codes, scales, W.data, Y)), "matmul_i8")
    return Y


def linear_i8(X, W: I8Weight, Y=None):
    """Y [T, N] = X W with X [T, K] (bf16) quantised per token on the way."""
    T = X.shape[0]
    _expect(X, (T, W.K), _BF16, "X")
    Y = torch.empty((T, W.N), dtype=torch.bfloat16, device=X.device) if Y is None else Y
    _expect(Y, (T, W.N), _BF16, "Y")
    scratch = torch.empty(_size(int(lib().linear_i8_scratch(T, W.K, W.N)), "linear_i8"), dtype=torch.uint8, device=X.device)
    _check(lib().linear_i8(_ptr(X), T, _ptr(W.data), W.K, W.N, _ptr(Y), _ptr(scratch), _stream(X, W.data, Y)), "linear_i8")
    return Y


class GatedI8Context(_Handle):
    """The gated feed-forward block on int8 weights (see gated_i8_ctx in the header) for up to T tokens; Wgu [D, 2 F] and Wd [F, D] are bf16 and not needed
    after the constructor's work on the stream."""
    _destroy = "gated_i8_ctx_destroy"

    def __init__(self, T: int, Wgu, Wd, act: str = "silu"):
        F, D = Wd.shape
        self.T, self.D, self.F = T, D, F
        gate = _gate(act)
        h = ctypes.c_void_p()
        _expect(Wgu, (D, 2 * F), _BF16, "Wgu")
        _expect(Wd, (F, D), _BF16, "Wd")
        _check(lib().gated_i8_ctx_create(ctypes.byref(h), T, D, F, gate), "gated_i8_ctx_create")
        self._own(h)
        self.set_weights(Wgu, Wd)

    def set_weights(self, Wgu, Wd):
        _expect(Wgu, (self.D, 2 * self.F), _BF16, "Wgu")
        _expect(Wd, (self.F, self.D), _BF16, "Wd")
        _check(lib().gated_i8_set_weights(self._h, _ptr(Wgu), _ptr(Wd), _stream(Wgu, Wd)), "gated_i8_set_weights")

    def fwd(self, X, Y=None):
        """X [t, D] with any t up to T -> Y [t, D]."""
        t = X.shape[0]
        _expect(X, (t, self.D), _BF16, "X")
        Y = torch.empty_like(X) if Y is None else Y
        _expect(Y, (t, self.D), _BF16, "Y")
        _check(lib().gated_i8_fwd(self._h, _ptr(X), t, _ptr(Y), _stream(X, Y)), "gated_i8_fwd")
        return Y

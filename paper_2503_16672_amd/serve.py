"""ctypes binding of include/ffn24_serve.h: mx4 numbers, products and the gated block on mx4 weights, the mixture of experts for few tokens.

Like the binding of ffn24_block.h it only marshals arguments: torch allocates and owns the tensors, every call enqueues on torch's current stream, and what does
not fit is refused with ValueError (shapes, types, contiguity, the device, checked here) or Ffn24Error (checked by the library).
"""
from __future__ import annotations

import ctypes

import torch

from . import ffn24
from .block import _NORM_TYPES, _Handle, _gate, _size, _stream
from .ffn24 import _BF16, _F32, _check, _expect, _ptr

EXPORTS = ("quantise_mx4", "dequantise_mx4", "mx4_weight_bytes", "mx4_weight", "mx4_weight_codes", "linear_mx4_scratch", "linear_mx4", "gated_mx4_ctx_create",
           "gated_mx4_ctx_destroy", "gated_mx4_set_weights", "gated_mx4_fwd", "moe_ctx_create", "moe_ctx_destroy", "moe_set_weights", "moe_fwd")

_lib = None


def lib() -> ctypes.CDLL:
    """libffn24.so with the argument types of this part of it."""
    global _lib
    if _lib is None:
        L = ffn24.lib()
        vp, i64, ci = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int
        L.quantise_mx4.argtypes = [vp, i64, i64, ci, vp, vp, vp]
        L.dequantise_mx4.argtypes = [vp, vp, i64, i64, ci, vp, vp]
        L.mx4_weight_bytes.argtypes = [i64, i64]
        L.mx4_weight.argtypes = [vp, i64, i64, ci, vp, vp]
        L.mx4_weight_codes.argtypes = [vp, vp, i64, i64, ci, vp, vp]
        L.linear_mx4_scratch.argtypes = [i64, i64, i64]
        L.linear_mx4.argtypes = [vp, i64, vp, i64, i64, vp, vp, vp]
        L.gated_mx4_ctx_create.argtypes = [ctypes.POINTER(vp), i64, i64, i64, ci]
        L.gated_mx4_ctx_destroy.argtypes = [vp]
        L.gated_mx4_set_weights.argtypes = [vp, vp, vp, vp]
        L.gated_mx4_fwd.argtypes = [vp, vp, i64, vp, vp]
        L.moe_ctx_create.argtypes = [ctypes.POINTER(vp), i64, i64, i64, i64, i64, ci, ci, ci]
        L.moe_ctx_destroy.argtypes = [vp]
        L.moe_set_weights.argtypes = [vp, vp, vp, vp, vp]
        L.moe_fwd.argtypes = [vp, vp, i64, vp, vp, vp, vp]
        for name in EXPORTS:
            getattr(L, name).restype = ci
        L.mx4_weight_bytes.restype = L.linear_mx4_scratch.restype = i64
        _lib = L
    return _lib


# ---------------------------------------------------------------------------------------------- mx4 numbers
_U8, _I32 = (torch.uint8,), (torch.int32,)


def _blocks(K: int) -> int:
    if K < 32 or K % 32:
        raise ValueError(f"{K} values a row, expected a multiple of 32")
    return K // 32


def quantise_mx4(X, codes=None, scales=None):
    """X [T, K] (bf16 or fp32) -> (codes [T, K / 2], scale codes [T, K / 32]), both uint8: 4-bit values, two a byte, and the power of two of each 32 of a row."""
    T, K = X.shape
    n = _blocks(K)
    _expect(X, (T, K), _NORM_TYPES, "X")
    codes = torch.empty((T, K // 2), dtype=torch.uint8, device=X.device) if codes is None else codes
    scales = torch.empty((T, n), dtype=torch.uint8, device=X.device) if scales is None else scales
    _expect(codes, (T, K // 2), _U8, "codes")
    _expect(scales, (T, n), _U8, "scales")
    _check(lib().quantise_mx4(_ptr(X), T, K, _NORM_TYPES[X.dtype], _ptr(codes), _ptr(scales), _stream(X, codes, scales)), "quantise_mx4")
    return codes, scales


def dequantise_mx4(codes, scales, Y=None, dtype=torch.bfloat16):
    """The values [T, K] that codes and scales stand for, in bf16 or fp32 (the type of Y if it is given)."""
    T, K = codes.shape[0], 2 * codes.shape[1]
    n = _blocks(K)
    _expect(codes, (T, K // 2), _U8, "codes")
    _expect(scales, (T, n), _U8, "scales")
    if Y is None and dtype not in _NORM_TYPES:
        raise ValueError(f"dtype: {dtype}, expected one of {tuple(_NORM_TYPES)}")
    Y = torch.empty((T, K), dtype=dtype, device=codes.device) if Y is None else Y
    _expect(Y, (T, K), _NORM_TYPES, "Y")
    _check(lib().dequantise_mx4(_ptr(codes), _ptr(scales), T, K, _NORM_TYPES[Y.dtype], _ptr(Y), _stream(codes, scales, Y)), "dequantise_mx4")
    return Y


class Mx4Weight:
    """W [K, N] (bf16) as mx4, blocks along K, laid out for linear_mx4; W is not needed afterwards."""

    def __init__(self, W):
        K, N = W.shape
        _expect(W, (K, N), _BF16, "W")
        self._make(K, N, W.device)
        _check(lib().mx4_weight(_ptr(W), K, N, 0, _ptr(self.data), _stream(W)), "mx4_weight")

    def _make(self, K, N, device):
        self.K, self.N = K, N
        self.data = torch.empty(_size(int(lib().mx4_weight_bytes(K, N)), "mx4_weight"), dtype=torch.uint8, device=device)

    @classmethod
    def from_codes(cls, codes, scales):
        """Of weights that are mx4 already: codes [N, K / 2] and scales [N, K / 32], a row an output channel, as quantise_mx4 makes them of W.T."""
        N, K = codes.shape[0], 2 * codes.shape[1]
        n = _blocks(K)
        _expect(codes, (N, K // 2), _U8, "codes")
        _expect(scales, (N, n), _U8, "scales")
        self = cls.__new__(cls)
        self._make(K, N, codes.device)
        _check(lib().mx4_weight_codes(_ptr(codes), _ptr(scales), K, N, 0, _ptr(self.data), _stream(codes, scales)), "mx4_weight_codes")
        return self


def linear_mx4(X, W: Mx4Weight, Y=None):
    """Y [T, N] = X W with X [T, K] (bf16) to mx4 on the way."""
    T = X.shape[0]
    _expect(X, (T, W.K), _BF16, "X")
    Y = torch.empty((T, W.N), dtype=torch.bfloat16, device=X.device) if Y is None else Y
    _expect(Y, (T, W.N), _BF16, "Y")
    L = lib()
    need = _size(int(L.linear_mx4_scratch(T, W.K, W.N)), "linear_mx4")
    scratch = torch.empty(need, dtype=torch.uint8, device=X.device) if need else None
    _check(L.linear_mx4(_ptr(X), T, _ptr(W.data), W.K, W.N, _ptr(Y), _ptr(scratch), _stream(X, W.data, Y)), "linear_mx4")
    return Y


# ---------------------------------------------------------------------------------------------- contexts
class GatedMx4Context(_Handle):
    """The gated feed-forward block on mx4 weights (see gated_mx4_ctx in the header) for up to T tokens; Wgu [D, 2 F] and Wd [F, D] are bf16 and not needed after the
    constructor's work on the stream."""
    _destroy = "gated_mx4_ctx_destroy"

    def __init__(self, T: int, Wgu, Wd, act: str = "silu"):
        F, D = Wd.shape
        self.T, self.D, self.F = T, D, F
        gate = _gate(act)
        h = ctypes.c_void_p()
        _expect(Wgu, (D, 2 * F), _BF16, "Wgu")
        _expect(Wd, (F, D), _BF16, "Wd")
        _check(lib().gated_mx4_ctx_create(ctypes.byref(h), T, D, F, gate), "gated_mx4_ctx_create")
        self._own(h)
        self.set_weights(Wgu, Wd)

    def set_weights(self, Wgu, Wd):
        _expect(Wgu, (self.D, 2 * self.F), _BF16, "Wgu")
        _expect(Wd, (self.F, self.D), _BF16, "Wd")
        _check(lib().gated_mx4_set_weights(self._h, _ptr(Wgu), _ptr(Wd), _stream(Wgu, Wd)), "gated_mx4_set_weights")

    def fwd(self, X, Y=None):
        """X [t, D] with any t up to T -> Y [t, D]."""
        t = X.shape[0]
        _expect(X, (t, self.D), _BF16, "X")
        Y = torch.empty_like(X) if Y is None else Y
        _expect(Y, (t, self.D), _BF16, "Y")
        _check(lib().gated_mx4_fwd(self._h, _ptr(X), t, _ptr(Y), _stream(X, Y)), "gated_mx4_fwd")
        return Y


EXPERTS = {"bf16": 0, "mx4": 1}


class MoeContext(_Handle):
    """A mixture of gated blocks (see moe_ctx in the header) for up to T <= 64 tokens a call: k of the E experts a token.  Wr [D, E], Wgu [E, D, 2 F] and Wd [E, F, D] are
    bf16 and not needed after the constructor's work on the stream; weights: the type the experts are kept in, "bf16" or "mx4"."""
    _destroy = "moe_ctx_destroy"

    def __init__(self, T: int, Wr, Wgu, Wd, k: int, act: str = "silu", renormalise: bool = True, weights: str = "bf16"):
        E, F, D = Wd.shape
        self.T, self.D, self.F, self.E, self.k = T, D, F, E, k
        gate = _gate(act)
        if weights not in EXPERTS:
            raise ValueError(f"weights: {weights!r}, expected one of {tuple(EXPERTS)}")
        h = ctypes.c_void_p()
        self._expect_weights(Wr, Wgu, Wd)
        _check(lib().moe_ctx_create(ctypes.byref(h), T, D, F, E, k, gate, int(renormalise), EXPERTS[weights]), "moe_ctx_create")
        self._own(h)
        self.set_weights(Wr, Wgu, Wd)

    def _expect_weights(self, Wr, Wgu, Wd):
        _expect(Wr, (self.D, self.E), _BF16, "Wr")
        _expect(Wgu, (self.E, self.D, 2 * self.F), _BF16, "Wgu")
        _expect(Wd, (self.E, self.F, self.D), _BF16, "Wd")

    def set_weights(self, Wr, Wgu, Wd):
        self._expect_weights(Wr, Wgu, Wd)
        _check(lib().moe_set_weights(self._h, _ptr(Wr), _ptr(Wgu), _ptr(Wd), _stream(Wr, Wgu, Wd)), "moe_set_weights")

    def fwd(self, X, Y=None, experts=None, shares=None):
        """X [t, D] with any t up to T -> Y [t, D].  experts [t, k] (int32) and shares [t, k] (fp32), given together, receive what the router chose."""
        t = X.shape[0]
        _expect(X, (t, self.D), _BF16, "X")
        Y = torch.empty_like(X) if Y is None else Y
        _expect(Y, (t, self.D), _BF16, "Y")
        _expect(experts, (t, self.k), _I32, "experts")
        _expect(shares, (t, self.k), _F32, "shares")
        _check(lib().moe_fwd(self._h, _ptr(X), t, _ptr(Y), _ptr(experts), _ptr(shares), _stream(X, Y, experts, shares)), "moe_fwd")
        return Y

"""Binding of the layer of experts for a few tokens (``include/hgemm_few_tokens.h``).  Argument marshalling only.

    layer = few_tokens.Layer(ctx, hidden=2048, inner=1024, experts=64, top_k=8, weights="nvfp4", activation="swiglu", dtype=torch.bfloat16)
    scratch = layer.empty_scratch(tokens)
    router.forward(logits, weights, indices)                      # routing.Router
    layer.run(x, w1, w2, indices, weights, y, scratch)            # w1, w2: (values, scale tiles, factors) of fp4.quantize_rows, or 16-bit stacks
"""
from __future__ import annotations

import ctypes

import torch

from . import fp4, hgemm
from .fp8 import TYPES, _dense, _ld, _stream

WEIGHTS = {"f16": 1, "bf16": 2, "nvfp4": 16, "mxfp4": 17}
ACTIVATIONS = {"silu": 0, "swiglu": 1}
MAX_TOKENS = 64

# every symbol include/hgemm_few_tokens.h declares
EXPORTS = ["hgemm_few_tokens_scratch", "hgemm_few_tokens"]


class Description(ctypes.Structure):
    """Mirror of ``hgemm_few_tokens_t``."""
    _fields_ = [("hidden", ctypes.c_int32), ("inner", ctypes.c_int32), ("experts", ctypes.c_int32), ("top_k", ctypes.c_int32), ("weights", ctypes.c_int32),
                ("activation", ctypes.c_int32), ("type", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class Weights(ctypes.Structure):
    """Mirror of ``hgemm_expert_weights_t``."""
    _fields_ = [("values", ctypes.c_void_p), ("ld", ctypes.c_int64), ("scales", ctypes.c_void_p), ("factor", ctypes.c_void_p)]


_lib = None


def lib() -> ctypes.CDLL:
    """The library (``hgemm.lib()``) with this header's signatures."""
    global _lib
    if _lib is None:
        L = hgemm.lib()
        i32, i64, p = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p
        dp, wp = ctypes.POINTER(Description), ctypes.POINTER(Weights)
        sig = {
            "hgemm_few_tokens_scratch": (i64, [dp, i64]),
            "hgemm_few_tokens": (i32, [p, dp, i64, p, i64, wp, wp, p, p, p, i64, p, i64, p]),
        }
        for name, (res, args) in sig.items():
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _lib = L
    return _lib


class Layer:
    """One layer's extents and types, and its calls.  weights: "f16" or "bf16" (w1 and w2 are stacks of matrices of x's type), "nvfp4" or "mxfp4" (tuples of
    packed values, scale tiles and, for "nvfp4", factors).  activation: "silu" (w1: experts x inner x hidden) or "swiglu" (experts x 2 inner x
    hidden, the gate's rows first); w2: experts x hidden x inner."""

    def __init__(self, ctx, hidden: int, inner: int, experts: int, top_k: int, weights: str = "nvfp4", activation: str = "swiglu", dtype=torch.bfloat16):
        if weights not in WEIGHTS or activation not in ACTIVATIONS:
            raise ValueError(f"weights is one of {', '.join(WEIGHTS)}, activation one of {', '.join(ACTIVATIONS)}")
        if dtype not in (torch.float16, torch.bfloat16):
            raise ValueError("x and y are float16 or bfloat16")
        self.ctx, self.dtype, self.weights, self._types = ctx, dtype, weights, (dtype,)
        self.hidden, self.inner, self.experts, self.top_k = int(hidden), int(inner), int(experts), int(top_k)
        self._desc = Description(self.hidden, self.inner, self.experts, self.top_k, WEIGHTS[weights], ACTIVATIONS[activation], TYPES[dtype], 0)
        self._ref = ctypes.byref(self._desc)
        self._call = lib().hgemm_few_tokens
        if lib().hgemm_few_tokens_scratch(self._ref, 0) < 0:
            raise ValueError(f"not a layer that can be run: {[getattr(self._desc, n) for n, _ in Description._fields_]}")
        self._w1 = torch.Size((self.experts, self.inner * (2 if activation == "swiglu" else 1), self.hidden))
        self._w2 = torch.Size((self.experts, self.hidden, self.inner))
        self._shapes = tuple((fp4._values_shape(s), fp4._scales_shape(s, weights)) for s in (self._w1, self._w2)) if weights in fp4.FORMATS else None

    def scratch_bytes(self, tokens: int) -> int:
        n = int(lib().hgemm_few_tokens_scratch(self._ref, tokens))
        if n < 0:
            raise ValueError(f"0 to {MAX_TOKENS} tokens, not {tokens}")
        return n

    def empty_scratch(self, tokens: int = MAX_TOKENS, device="cuda"):
        """Scratch memory for calls of up to `tokens` tokens; calls that may overlap take one each."""
        return torch.empty(max(16, self.scratch_bytes(tokens)), dtype=torch.uint8, device=device)

    def _weights(self, w, i, name):
        if self._shapes is None:
            shape = (self._w1, self._w2)[i]
            return Weights(w.data_ptr(), _ld(w, shape, (self.dtype,), name), None, None)
        if len(w) not in (2, 3):
            raise ValueError(f"{name} must be (values, scale tiles, factors)")
        values, tiles = self._shapes[i]
        v = w[0]
        st = v.stride()
        if len(st) == 3 and st[2] == 1 and st[1] >= values[2] > 1 and st[1] % 16 == 0 and st[0] == values[1] * st[1] and v.shape == values and v.dtype == torch.uint8 and v.is_cuda:
            ld = st[1]                                            # matrices one after the other, as fp4.empty_rows makes them
        else:
            ld = fp4._ld_bytes(v, values, name)
        factor = fp4._factor_of(w[2] if len(w) == 3 else None, self.experts, self.weights, f"{name} factors")
        return Weights(v.data_ptr(), ld, _dense(w[1], tiles, torch.uint8, name), factor)

    def run(self, x, w1, w2, indices, weights, y, scratch, stream=None) -> None:
        """y (T, hidden) = the layer on x (T, hidden); indices (T, top_k) int32 and weights (T, top_k) fp32 are a router's."""
        T = x.shape[0]
        shape, chosen = (T, self.hidden), (T, self.top_k)
        ldx, ldy = _ld(x, shape, self._types, "x"), _ld(y, shape, self._types, "y")
        i, w = _dense(indices, chosen, torch.int32, "indices"), _dense(weights, chosen, torch.float32, "weights")
        s = _dense(scratch, scratch.shape, torch.uint8, "scratch")
        a, b = self._weights(w1, 0, "w1"), self._weights(w2, 1, "w2")
        st = self._call(self.ctx._h, self._ref, T, x.data_ptr(), ldx, ctypes.byref(a), ctypes.byref(b), i, w, y.data_ptr(), ldy, s, scratch.numel(), _stream(self.ctx, stream))
        if st != hgemm.OK:
            raise hgemm.HgemmError(st, f"hgemm_few_tokens({T} tokens, {self.weights})")

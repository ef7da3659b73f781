"""Binding of the routing to experts (``include/hgemm_routing.h``).  Argument marshalling only.

    router = routing.Router(ctx, experts=64, top_k=8, score="sigmoid", renormalize=True)
    router.forward(logits, weights, indices, bias=bias)           # (T, 64) -> (T, 8) fp32 and int32
    router.sort(indices, offsets, order, position)                # expert order of the T * 8 choices
    router.backward(logits, indices, dweights, dlogits)
"""
from __future__ import annotations

import ctypes

import torch

from . import fp8, hgemm
from .fp8 import _check, _dense, _ld, _stream

SCORES = {"softmax": 0, "sigmoid": 1}
GROUP_SCORES = {"max": 0, "top2": 1}
_WIDE = (torch.float32, torch.float16, torch.bfloat16)

# every symbol include/hgemm_routing.h declares
EXPORTS = ["hgemm_route", "hgemm_route_backward", "hgemm_route_sort"]


class Routing(ctypes.Structure):
    """Mirror of ``hgemm_routing_t``."""
    _fields_ = [("experts", ctypes.c_int32), ("top_k", ctypes.c_int32), ("score", ctypes.c_int32), ("groups", ctypes.c_int32), ("top_groups", ctypes.c_int32),
                ("group_score", ctypes.c_int32), ("renormalize", ctypes.c_int32), ("scale", ctypes.c_float)]


_lib = None


def lib() -> ctypes.CDLL:
    global _lib
    if _lib is None:
        L = hgemm.lib()
        i32, i64, p = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p
        rp = ctypes.POINTER(Routing)
        sig = {
            "hgemm_route": (i32, [p, rp, i64, p, i32, i64, p, p, p, p]),
            "hgemm_route_backward": (i32, [p, rp, i64, p, i32, i64, p, p, p, i64, p]),
            "hgemm_route_sort": (i32, [p, p, i64, i32, p, p, p, p]),
        }
        for name, (res, args) in sig.items():
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _lib = L
    return _lib


class Router:
    """One router's rule (see ``include/hgemm_routing.h``) and its calls."""

    def __init__(self, ctx, experts: int, top_k: int, score: str = "softmax", groups: int = 1, top_groups: int = 1, group_score: str = "max",
                 renormalize: bool = True, scale: float = 1.0):
        if score not in SCORES or group_score not in GROUP_SCORES:
            raise ValueError(f"score is one of {', '.join(SCORES)}, group_score one of {', '.join(GROUP_SCORES)}")
        self.ctx = ctx
        self.experts, self.top_k = int(experts), int(top_k)
        self._desc = Routing(self.experts, self.top_k, SCORES[score], int(groups), int(top_groups), GROUP_SCORES[group_score], 1 if renormalize else 0, float(scale))
        self._ref = ctypes.byref(self._desc)
        _check(lib().hgemm_route(ctx._h, self._ref, 0, None, 0, self.experts, 1, None, None, None), f"hgemm_route{self.rule}")       # the rule's own checks; no tokens

    @property
    def rule(self) -> tuple:
        return tuple(getattr(self._desc, n) for n, _ in Routing._fields_)

    def _rows(self, t, name):
        if t.dim() != 2 or t.shape[1] != self.experts:
            raise ValueError(f"{name} must be tokens x {self.experts}")
        return _ld(t, t.shape, _WIDE, name)

    def forward(self, logits, weights, indices, bias=None, stream=None) -> None:
        """weights (T, top_k) fp32 and indices (T, top_k) int32 of the chosen experts, best first."""
        ld, T = self._rows(logits, "logits"), logits.shape[0]
        w, i = _dense(weights, (T, self.top_k), torch.float32, "weights"), _dense(indices, (T, self.top_k), torch.int32, "indices")
        b = None if bias is None else _dense(bias, (self.experts,), torch.float32, "bias")
        _check(lib().hgemm_route(self.ctx._h, self._ref, T, logits.data_ptr(), fp8.TYPES[logits.dtype], ld, b, w, i, _stream(self.ctx, stream)), f"hgemm_route{self.rule}")

    def backward(self, logits, indices, dweights, dlogits, stream=None) -> None:
        """dlogits (T, experts), of the logits' type, from dweights (T, top_k) fp32."""
        ld, T = self._rows(logits, "logits"), logits.shape[0]
        ldd = self._rows(dlogits, "dlogits")
        if dlogits.dtype != logits.dtype or dlogits.shape != logits.shape:
            raise ValueError("dlogits must have the shape and type of logits")
        i, d = _dense(indices, (T, self.top_k), torch.int32, "indices"), _dense(dweights, (T, self.top_k), torch.float32, "dweights")
        _check(lib().hgemm_route_backward(self.ctx._h, self._ref, T, logits.data_ptr(), fp8.TYPES[logits.dtype], ld, i, d, dlogits.data_ptr(), ldd, _stream(self.ctx, stream)),
               f"hgemm_route_backward{self.rule}")

    def sort(self, indices, offsets, order, position, stream=None) -> None:
        """Expert order of the choices (int32 throughout): offsets (experts + 1), order and position (T * top_k)."""
        n = indices.numel()
        i = _dense(indices, indices.shape, torch.int32, "indices")
        o, r, p = _dense(offsets, (self.experts + 1,), torch.int32, "offsets"), _dense(order, (n,), torch.int32, "order"), _dense(position, (n,), torch.int32, "position")
        _check(lib().hgemm_route_sort(self.ctx._h, i, n, self.experts, o, r, p, _stream(self.ctx, stream)), f"hgemm_route_sort({n} choices, {self.experts} experts)")

"""Binding of the 4-bit products with block scales (``include/hgemm_fp4.h``): quantisation, products of a linear layer,
products over experts.  Argument marshalling only; see ``hgemm.py`` for the conventions (context, streams, errors).

    q, s = fp4.empty_rows(M, K)                       # packed values (two to a byte, rows at multiples of 16 bytes) and scale tiles
    f = torch.empty(1, device="cuda")                 # the tensor's factor ("nvfp4" only)
    fp4.tensor_factor(ctx, x, f)
    fp4.quantize_rows(ctx, x, q, s, factor=f)
    wq, ws = fp4.empty_rows(N, K)
    fp4.tensor_factor(ctx, w, wf)
    fp4.quantize_rows(ctx, w, wq, ws, factor=wf)
    plan = fp4.Plan(ctx, M, N, K, form="forward", out_dtype=torch.bfloat16)
    plan.run(q, s, wq, ws, y, a_factor=f, b_factor=wf)

format="mxfp4": blocks of 32 with powers of two and no factor.
"""
from __future__ import annotations

import ctypes

import torch

from . import fp8, hgemm
from .fp8 import FORMS, TYPES, _WIDE, _check, _dense, _groups_of, _ld, _source, _stream, padded_rows
from .hgemm import OK, HgemmError

FORMATS = {"nvfp4": 0, "mxfp4": 1}
BLOCK = {"nvfp4": 16, "mxfp4": 32}
ROWS, COLS = 1, 2
TILE_ROWS, TILE_BYTES = 128, 512
#: What the 16 codes stand for.
VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0)

# every symbol include/hgemm_fp4.h declares
EXPORTS = ["hgemm_fp4_scale_bytes", "hgemm_fp4_tensor_factor", "hgemm_fp4_quantize", "hgemm_fp4_dequantize", "hgemm_fp4_plan", "hgemm_fp4_plan_destroy", "hgemm_fp4_run",
           "hgemm_fp4_last_device_status", "hgemm_fp4_debug_timeout_probe", "hgemm_fp4_plan_get_config", "hgemm_fp4_plan_set_config", "hgemm_fp4_planned_config"]


class Quantize(ctypes.Structure):
    """Mirror of ``hgemm_fp4_quantize_t``."""
    _fields_ = [("blocks", ctypes.c_int32), ("x_type", ctypes.c_int32), ("format", ctypes.c_int32), ("matrices", ctypes.c_int32), ("rows", ctypes.c_int64),
                ("cols", ctypes.c_int64), ("ldx", ctypes.c_int64), ("x", ctypes.c_void_p), ("row_index", ctypes.c_void_p), ("x_rows", ctypes.c_int64),
                ("offsets", ctypes.c_void_p), ("groups", ctypes.c_int32), ("reserved", ctypes.c_int32), ("factor", ctypes.c_void_p), ("q", ctypes.c_void_p),
                ("ldq", ctypes.c_int64), ("scales", ctypes.c_void_p), ("q_cols", ctypes.c_void_p), ("ldq_cols", ctypes.c_int64), ("scales_cols", ctypes.c_void_p)]


class Config(ctypes.Structure):
    """Mirror of ``hgemm_fp4_config_t``."""
    _fields_ = [("cta_group", ctypes.c_int32), ("block_q", ctypes.c_int32), ("split_k", ctypes.c_int32), ("reserved", ctypes.c_int32)]

    def as_dict(self) -> dict:
        return {k: int(getattr(self, k)) for k, _ in self._fields_ if k != "reserved"}


_lib = None


def lib() -> ctypes.CDLL:
    """The library (``hgemm.lib()``) with this header's signatures."""
    global _lib
    if _lib is None:
        L = hgemm.lib()
        fp8.lib()
        i32, i64, p = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p
        cfgp = ctypes.POINTER(Config)
        sig = {
            "hgemm_fp4_scale_bytes": (i64, [i64, i64, i32]),
            "hgemm_fp4_tensor_factor": (i32, [p, i32, i64, i64, i64, p, i64, p, p]),
            "hgemm_fp4_quantize": (i32, [p, ctypes.POINTER(Quantize), p]),
            "hgemm_fp4_dequantize": (i32, [p, i32, i32, i64, i64, i64, p, i64, p, p, p, i32, p, i64, p]),
            "hgemm_fp4_plan": (i32, [p, i32, i64, i64, i64, i32, i32, i32, ctypes.POINTER(p)]),
            "hgemm_fp4_plan_destroy": (i32, [p]),
            "hgemm_fp4_run": (i32, [p, p, i64, p, p, p, i64, p, p, p, i64, p, i32, p]),
            "hgemm_fp4_last_device_status": (i32, [p, ctypes.POINTER(ctypes.c_uint32)]),
            "hgemm_fp4_debug_timeout_probe": (i32, [p, p]),
            "hgemm_fp4_plan_get_config": (i32, [p, cfgp]),
            "hgemm_fp4_plan_set_config": (i32, [p, cfgp]),
            "hgemm_fp4_planned_config": (i32, [i32, i64, i64, i64, i32, i32, cfgp]),
        }
        for name, (res, args) in sig.items():
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _lib = L
    return _lib


def planned_config(form: str, M: int, N: int, K: int, groups: int = 0, num_sms: int = 148) -> Config:
    c = Config()
    _check(lib().hgemm_fp4_planned_config(FORMS[form], M, N, K, groups, num_sms, ctypes.byref(c)), f"hgemm_fp4_planned_config({form},{M},{N},{K},{groups})")
    return c


# ---- buffers -------------------------------------------------------------------------------------

def _up(n: int, unit: int) -> int:
    return -(-n // unit)


def _format(format: str) -> int:
    if format not in FORMATS:
        raise ValueError(f"format must be one of {', '.join(FORMATS)}")
    return FORMATS[format]


def _values_shape(shape):
    return (*shape[:-1], -(-shape[-1] // 2))


def _scales_shape(shape, format):
    return (*shape[:-2], -(-shape[-2] // TILE_ROWS), -(-shape[-1] // (4 * BLOCK[format])), TILE_BYTES)


def _col_shape(shape, groups):
    """The column copy's extents: the transposed matrix, laid out per group where there are groups."""
    return (*shape[:-2], shape[-1], padded_rows(shape[-2], groups) if groups else shape[-2])


def _empty(shape, scale_shape, format, device):
    pitch = _up(shape[-1], 32) * 16
    values = torch.empty(*shape[:-1], pitch, dtype=torch.uint8, device=device)[..., :_up(shape[-1], 2)]
    return values, torch.empty(_scales_shape(scale_shape, format), dtype=torch.uint8, device=device)


def empty_rows(*shape, format: str = "nvfp4", groups: int = 0, device="cuda"):
    """Uninitialised (values, scale tiles) of a row copy: shape (R, C), or (matrices, R, C); groups > 0: scale tiles per group."""
    _format(format)
    return _empty(shape, (padded_rows(shape[0], groups), shape[1]) if groups else shape, format, device)


def empty_cols(*shape, format: str = "nvfp4", groups: int = 0, device="cuda"):
    """Uninitialised (values, scale tiles) of the column copy of a matrix, or of a stack, of that shape; groups > 0: laid out per group."""
    _format(format)
    s = _col_shape(shape, groups)
    return _empty(s, s, format, device)


def scale_matrix(scales, rows: int, cols: int, format: str = "nvfp4"):
    """The scales of scale tiles as a matrix (..., rows, blocks): torch.float8_e4m3fn ("nvfp4") or exponents as uint8 ("mxfp4")."""
    _format(format)
    s = scales.unflatten(-1, (32, 4, 4))                          # (..., tiles, atoms, row, quarter, block)
    n = s.dim() - 5
    s = s.permute(*range(n), n, n + 3, n + 2, n + 1, n + 4)
    s = s.reshape(*scales.shape[:-3], scales.shape[-3] * TILE_ROWS, scales.shape[-2] * 4)[..., :rows, :_up(cols, BLOCK[format])]
    return s.contiguous().view(torch.float8_e4m3fn) if format == "nvfp4" else s


# ---- quantisation --------------------------------------------------------------------------------

def _ld_bytes(t, shape, name):
    ld = _ld(t, shape, (torch.uint8,), name)
    if t.numel() == 0:                                            # no rows, or rows of nothing
        return -(-max(shape[-1], 1) // 16) * 16
    if ld % 16:
        raise ValueError(f"{name}: rows must be multiples of 16 bytes apart, not {ld}")
    return ld


def _factor_of(factor, n: int, format: str, name: str = "factor"):
    if format != "nvfp4":
        if factor is not None:
            raise ValueError(f"{name}: {format} has no factor")
        return None
    if factor is None:
        raise ValueError(f"{name}: nvfp4 needs the tensor's factor")
    return _dense(factor, (n,), torch.float32, name)


def _copy(q, s, shape, scale_shape, format, name):
    """The pointers' arguments of a copy: (values, bytes between rows, scales)."""
    ld = _ld_bytes(q, _values_shape(shape), name)
    return q.data_ptr(), ld, _dense(s, _scales_shape(scale_shape, format), torch.uint8, name + " scales")


def _matrix(x):
    """(matrices, rows, cols, ld) of a matrix or a stack."""
    if x.dim() not in (2, 3):
        raise ValueError("x must be a matrix or a stack of matrices")
    return (x.shape[0] if x.dim() == 3 else 1), x.shape[-2], x.shape[-1], _ld(x, x.shape, _WIDE, "x")


def tensor_factor(ctx, x, factor, stream=None) -> None:
    """factor (1,), or (matrices,) for a stack: the "nvfp4" factor of x (fp32, fp16 or bf16), max |x| / 2688 rounded up to a power of two."""
    n, R, C, ld = _matrix(x)
    f = _dense(factor, (n,), torch.float32, "factor")
    st = lib().hgemm_fp4_tensor_factor(ctx._h, TYPES[x.dtype], n, R, C, x.data_ptr(), ld, f, _stream(ctx, stream))
    if st != OK:
        raise HgemmError(st, f"hgemm_fp4_tensor_factor({tuple(x.shape)})")


def _quantize(ctx, x, row_copy, col_copy, factor, format, rows, offsets, stream):
    fmt = _format(format)
    if x.dim() == 3:
        if rows is not None or offsets is not None:
            raise ValueError("a stack is quantised without rows and offsets")
        n, R, C, ld = _matrix(x)
    else:
        R, C, ld = _source(x, rows)
        n = 1
    shape = (*x.shape[:-2], R, C)
    groups = _groups_of(offsets)
    place = (padded_rows(R, groups), C) if groups else shape
    f = _factor_of(factor, n, format)
    q, ldq, s = (None, 0, None) if row_copy is None else _copy(*row_copy, shape, place, format, "q")
    cols = _col_shape(shape, groups)
    qc, ldqc, sc = (None, 0, None) if col_copy is None else _copy(*col_copy, cols, cols, format, "q_cols")
    d = Quantize((ROWS if row_copy is not None else 0) | (COLS if col_copy is not None else 0), TYPES[x.dtype], fmt, n, R, C, ld, x.data_ptr(),
                 None if rows is None else rows.data_ptr(), x.shape[-2], None if offsets is None else offsets.data_ptr(), groups, 0, f, q, ldq, s, qc, ldqc, sc)
    st = lib().hgemm_fp4_quantize(ctx._h, ctypes.byref(d), _stream(ctx, stream))
    if st != OK:
        raise HgemmError(st, f"hgemm_fp4_quantize(blocks={d.blocks}, {R}x{C})")


def quantize_rows(ctx, x, q, scales, factor=None, format: str = "nvfp4", rows=None, offsets=None, stream=None) -> None:
    """The row copy of x (fp32, fp16 or bf16 matrix, or a stack of weights); rows: int32 row numbers, row r of the result is row rows[r] of x (a row of
    zeros for a number outside it); offsets: scale tiles per group (see ``empty_rows``)."""
    _quantize(ctx, x, (q, scales), None, factor, format, rows, offsets, stream)


def quantize_cols(ctx, x, q, scales, factor=None, format: str = "nvfp4", rows=None, offsets=None, stream=None) -> None:
    """The column copy of x (the transposed matrix); offsets: laid out per group (see ``empty_cols``)."""
    _quantize(ctx, x, None, (q, scales), factor, format, rows, offsets, stream)


def quantize_both(ctx, x, q, scales, q_cols, scales_cols, factor=None, format: str = "nvfp4", rows=None, offsets=None, stream=None) -> None:
    """The row and the column copy in one pass over x."""
    _quantize(ctx, x, (q, scales), (q_cols, scales_cols), factor, format, rows, offsets, stream)


def dequantize(ctx, q, scales, out, factor=None, format: str = "nvfp4", offsets=None, stream=None) -> None:
    """out (fp32, fp16 or bf16; the copy's shape in elements) = what a copy stands for; offsets: of a row copy with scale tiles per group."""
    fmt = _format(format)
    if out.dim() not in (2, 3):
        raise ValueError("out must be a matrix or a stack of matrices")
    n, shape = (out.shape[0] if out.dim() == 3 else 1), out.shape
    ldo = _ld(out, shape, _WIDE, "out")
    groups = _groups_of(offsets)
    if groups and out.dim() == 3:
        raise ValueError("a stack has no offsets")
    v, ld, s = _copy(q, scales, shape, (padded_rows(shape[0], groups), shape[1]) if groups else shape, format, "q")
    st = lib().hgemm_fp4_dequantize(ctx._h, fmt, TYPES[out.dtype], n, shape[-2], shape[-1], v, ld, s, _factor_of(factor, n, format), None if offsets is None else offsets.data_ptr(),
                                    groups, out.data_ptr(), ldo, _stream(ctx, stream))
    if st != OK:
        raise HgemmError(st, f"hgemm_fp4_dequantize({tuple(shape)})")


# ---- products ------------------------------------------------------------------------------------

class Plan:
    """``hgemm_fp4_plan`` / ``hgemm_fp4_run``: one of a layer's three products.

    form "forward": run(x (M,K) row copy, w (N,K) row copy, y (M,N)); "input_grad": run(dy (M,N) row copy, w column copy (K,N), dx (M,K));
    "weight_grad": run(dy column copy (N,M), x column copy (K,M), dw (N,K)) -- each copy as values and scale tiles, and for "nvfp4" a factor.  groups > 0: one
    weight per group -- w a stack, dw (groups,N,K), ``offsets`` with every run, row copies with scale tiles per group, column copies of dy and x laid out per
    group.

    Each plan holds one of the context's 4095 status words until it is closed or dropped; a program keeps its plans."""

    def __init__(self, ctx, M: int, N: int, K: int, form: str = "forward", groups: int = 0, format: str = "nvfp4", out_dtype=torch.bfloat16):
        if form not in FORMS:
            raise ValueError(f"form must be one of {', '.join(FORMS)}")
        if out_dtype not in _WIDE:
            raise ValueError("results are float32, float16 or bfloat16")
        self.ctx = ctx
        self.shape = (int(M), int(N), int(K))
        self.form, self.groups, self.format = form, int(groups), format
        self._h = ctypes.c_void_p()
        self._run, self._destroy = lib().hgemm_fp4_run, lib().hgemm_fp4_plan_destroy
        _check(lib().hgemm_fp4_plan(ctx._h, FORMS[form], *self.shape, self.groups, _format(format), TYPES[out_dtype], ctypes.byref(self._h)),
               f"hgemm_fp4_plan({form},{M},{N},{K},groups={groups})")
        M, N, K = self.shape
        g = (self.groups,) if self.groups else ()
        rows = padded_rows(M, self.groups) if self.groups else M
        if form == "weight_grad":
            a, b, c = (N, rows), (K, rows), (*g, N, K)
            sa, sb = a, b
        else:
            d = K if form == "forward" else N
            a, b, c = (M, d), (*g, N + K - d, d), (M, N + K - d)
            sa, sb = (rows, d), b
        self._a, self._b, self._c = _values_shape(a), _values_shape(b), torch.Size(c)
        self._sa, self._sb = _scales_shape(sa, format), _scales_shape(sb, format)
        self._out = (out_dtype,)
        self._b_factors = self.groups if self.groups and form != "weight_grad" else 1

    @property
    def config(self) -> Config:
        c = Config()
        _check(lib().hgemm_fp4_plan_get_config(self._open(), ctypes.byref(c)), "hgemm_fp4_plan_get_config")
        return c

    def set_config(self, cta_group: int, block_q: int, split_k: int = 1) -> None:
        c = Config(cta_group, block_q, split_k, 0)
        _check(lib().hgemm_fp4_plan_set_config(self._open(), ctypes.byref(c)), f"hgemm_fp4_plan_set_config({c.as_dict()})")

    def _open(self):
        """The library's handle; none once the plan or its context is closed (the library then refuses the call)."""
        return self._h if self.ctx._h else None

    def last_device_status(self) -> tuple[int, int]:
        """``hgemm_fp4_last_device_status``: (status, code) of this plan's own status word; synchronises the device."""
        code = ctypes.c_uint32(0)
        st = lib().hgemm_fp4_last_device_status(self._open(), ctypes.byref(code))
        return int(st), int(code.value)

    def debug_timeout_probe(self, stream: int = 0) -> None:
        _check(lib().hgemm_fp4_debug_timeout_probe(self._open(), ctypes.c_void_p(stream)), "hgemm_fp4_debug_timeout_probe")

    def run(self, a, a_scales, b, b_scales, out, a_factor=None, b_factor=None, offsets=None, accumulate: bool = False, stream=None) -> None:
        lda, ldb, ldc = _ld_bytes(a, self._a, "a"), _ld_bytes(b, self._b, "b"), _ld(out, self._c, self._out, "out")
        sa, sb = _dense(a_scales, self._sa, torch.uint8, "a_scales"), _dense(b_scales, self._sb, torch.uint8, "b_scales")
        fa, fb = _factor_of(a_factor, 1, self.format, "a_factor"), _factor_of(b_factor, self._b_factors, self.format, "b_factor")
        off = None
        if self.groups:
            if offsets is None:
                raise ValueError("a plan with groups needs their offsets")
            off = _dense(offsets, (self.groups + 1,), torch.int32, "offsets")
        elif offsets is not None:
            raise ValueError("offsets belong to a plan with groups")
        st = self._run(self._open(), a.data_ptr(), lda, sa, fa, b.data_ptr(), ldb, sb, fb, out.data_ptr(), ldc, off, 1 if accumulate else 0, _stream(self.ctx, stream))
        if st != OK:
            raise HgemmError(st, f"hgemm_fp4_run({self.form}{self.shape}, groups={self.groups})")

    def close(self) -> None:
        if self._h and self.ctx._h:
            self._destroy(self._h)
        self._h = ctypes.c_void_p()

    def __del__(self):
        h = getattr(self, "_h", None)                  # none: the plan was never made.  No module's names: at exit they may be gone
        if h and self.ctx._h:
            self._destroy(h)

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

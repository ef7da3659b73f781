"""Binding of the 8-bit products with block scales (``include/hgemm_fp8.h``): quantisation, products of a linear layer,
products over experts.  Argument marshalling only; see ``hgemm.py`` for the conventions (context, streams, errors).

    q, s = fp8.empty_rows(M, K)                      # 8-bit values (rows start at multiples of 16 bytes) and scales
    fp8.quantize_rows(ctx, x, q, s)
    wq, ws = fp8.empty_tiles(N, K)
    fp8.quantize_tiles(ctx, w, wq, ws)
    plan = fp8.Plan(ctx, M, N, K, form="forward", out_dtype=torch.bfloat16)
    plan.run(q, s, wq, ws, y)
"""
from __future__ import annotations

import ctypes

import torch

from . import hgemm
from .hgemm import OK, HgemmError

BLOCK = 128
ROWS, COLS, TILES = 1, 2, 4
FORMS = {"forward": 0, "input_grad": 1, "weight_grad": 2}
TYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2, torch.float8_e4m3fn: 3, torch.float8_e5m2: 4}
_WIDE = (torch.float32, torch.float16, torch.bfloat16)
_FP8 = (torch.float8_e4m3fn, torch.float8_e5m2)

# every symbol include/hgemm_fp8.h declares
EXPORTS = ["hgemm_fp8_quantize", "hgemm_fp8_padded_rows", "hgemm_fp8_plan", "hgemm_fp8_plan_destroy", "hgemm_fp8_run", "hgemm_fp8_plan_get_config",
           "hgemm_fp8_plan_set_config", "hgemm_fp8_planned_config", "hgemm_fp8_last_device_status", "hgemm_fp8_debug_timeout_probe"]


class Quantize(ctypes.Structure):
    """Mirror of ``hgemm_fp8_quantize_t``."""
    _fields_ = [("blocks", ctypes.c_int32), ("x_type", ctypes.c_int32), ("q_type", ctypes.c_int32), ("pow2", ctypes.c_int32), ("rows", ctypes.c_int64),
                ("cols", ctypes.c_int64), ("ldx", ctypes.c_int64), ("x", ctypes.c_void_p), ("row_index", ctypes.c_void_p), ("x_rows", ctypes.c_int64),
                ("offsets", ctypes.c_void_p), ("groups", ctypes.c_int32), ("reserved", ctypes.c_int32), ("q", ctypes.c_void_p), ("ldq", ctypes.c_int64),
                ("scales", ctypes.c_void_p), ("q_cols", ctypes.c_void_p), ("ldq_cols", ctypes.c_int64), ("scales_cols", ctypes.c_void_p)]


class Config(ctypes.Structure):
    """Mirror of ``hgemm_fp8_config_t``."""
    _fields_ = [("cta_group", ctypes.c_int32), ("block_q", ctypes.c_int32), ("split_k", ctypes.c_int32), ("reserved", ctypes.c_int32)]

    def as_dict(self) -> dict:
        return {k: int(getattr(self, k)) for k, _ in self._fields_ if k != "reserved"}


_lib = None


def lib() -> ctypes.CDLL:
    """The library (``hgemm.lib()``) with this header's signatures."""
    global _lib
    if _lib is None:
        L = hgemm.lib()
        i32, i64, p = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p
        cfgp = ctypes.POINTER(Config)
        sig = {
            "hgemm_fp8_quantize": (i32, [p, ctypes.POINTER(Quantize), p]),
            "hgemm_fp8_padded_rows": (i64, [i64, i32]),
            "hgemm_fp8_plan": (i32, [p, i32, i64, i64, i64, i32, i32, i32, i32, ctypes.POINTER(p)]),
            "hgemm_fp8_plan_destroy": (i32, [p]),
            "hgemm_fp8_run": (i32, [p, p, i64, p, p, i64, p, p, i64, p, i32, p]),
            "hgemm_fp8_plan_get_config": (i32, [p, cfgp]),
            "hgemm_fp8_plan_set_config": (i32, [p, cfgp]),
            "hgemm_fp8_last_device_status": (i32, [p, ctypes.POINTER(ctypes.c_uint32)]),
            "hgemm_fp8_debug_timeout_probe": (i32, [p, p]),
            "hgemm_fp8_planned_config": (i32, [i32, i64, i64, i64, i32, i32, cfgp]),
        }
        for name, (res, args) in sig.items():
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _lib = L
    return _lib


def _check(status: int, what: str) -> None:
    if status != OK:
        raise HgemmError(status, what)


# the current stream's handle without building a Stream object (which costs more than the rest of a call)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda device: torch.cuda.current_stream(device).cuda_stream)


def _stream(ctx, stream) -> int:
    return _raw_stream(ctx.device) if stream is None else int(stream)


def padded_rows(M: int, groups: int) -> int:
    """Rows of a column-quantised copy laid out per group."""
    return int(lib().hgemm_fp8_padded_rows(int(M), int(groups)))


def planned_config(form: str, M: int, N: int, K: int, groups: int = 0, num_sms: int = 148) -> Config:
    c = Config()
    _check(lib().hgemm_fp8_planned_config(FORMS[form], M, N, K, groups, num_sms, ctypes.byref(c)), f"hgemm_fp8_planned_config({form},{M},{N},{K},{groups})")
    return c


# ---- buffers -------------------------------------------------------------------------------------

def _values(shape, dtype, device):
    pitch = -(-shape[-1] // 16) * 16
    return torch.empty(*shape[:-1], pitch, dtype=dtype, device=device)[..., :shape[-1]]


def _blocks(n: int) -> int:
    return -(-n // BLOCK)


def empty_rows(rows: int, cols: int, dtype=torch.float8_e4m3fn, device="cuda"):
    """Uninitialised (values, scales) for ``quantize_rows``."""
    return _values((rows, cols), dtype, device), torch.empty(rows, _blocks(cols), device=device)


def empty_cols(rows: int, cols: int, groups: int = 0, dtype=torch.float8_e4m3fn, device="cuda"):
    """Uninitialised (values, scales) for ``quantize_cols``; groups > 0: laid out per group."""
    r = padded_rows(rows, groups) if groups else rows
    return _values((r, cols), dtype, device), torch.empty(_blocks(r), cols, device=device)


def empty_tiles(*shape, dtype=torch.float8_e4m3fn, device="cuda"):
    """Uninitialised (values, scales) for ``quantize_tiles``: shape (N, K) or (groups, N, K)."""
    return _values(shape, dtype, device), torch.empty(*shape[:-2], _blocks(shape[-2]), _blocks(shape[-1]), device=device)


# ---- quantisation --------------------------------------------------------------------------------

def _dense(t, shape, dtype, name):
    if t.dtype == dtype and t.shape == shape and t.is_cuda and t.is_contiguous():
        return t.data_ptr()
    raise ValueError(f"{name} must be a contiguous CUDA {dtype} tensor of shape {tuple(shape)}, not {tuple(t.shape)} {t.dtype}")


def _ld(t, shape, dtypes, name):
    """Elements between the rows of a matrix, or of a stack of matrices that follow one another."""
    if t.dtype not in dtypes or t.shape != shape or not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor of shape {tuple(shape)} and type {' / '.join(str(d) for d in dtypes)}, not {tuple(t.shape)} {t.dtype}")
    st = t.stride()
    if len(st) == 2 and st[1] == 1 and st[0] >= shape[1] and shape[0] > 1:
        return st[0]
    if st[-1] != 1 and shape[-1] > 1:
        raise ValueError(f"{name}: the elements of a row must be consecutive")
    if len(shape) == 3 and shape[1] == 1 and shape[0] > 1:      # matrices of one row: the next row is the next matrix's
        if st[0] < shape[2]:
            raise ValueError(f"{name}: strides {st} are not those of row-major matrices one after the other")
        return st[0]
    # one row: its distance to a next one is free, any that the library accepts
    ld = max(st[-2], shape[-1]) if shape[-2] > 1 else -(-max(st[-2], shape[-1]) // 16) * 16
    if (shape[-2] > 1 and st[-2] < shape[-1]) or (len(shape) == 3 and shape[0] > 1 and st[0] != shape[1] * ld):
        raise ValueError(f"{name}: strides {st} are not those of row-major matrices one after the other")
    return ld


def _quantize(ctx, blocks, x, shape, ldx, row_index, x_rows, offsets, groups, pow2, by, by_cols, stream):
    q, s = by if by is not None else (None, None)
    qc, sc = by_cols if by_cols is not None else (None, None)
    dtype = (q if q is not None else qc).dtype
    if q is not None and qc is not None and q.dtype != qc.dtype:
        raise ValueError("row and column copies have the same type")
    rows, cols = shape
    d = Quantize(blocks, TYPES[x.dtype], TYPES[dtype], 1 if pow2 else 0, rows, cols, ldx, x.data_ptr(),
                 None if row_index is None else row_index.data_ptr(), x_rows, None if offsets is None else offsets.data_ptr(), groups, 0,
                 None if q is None else q.data_ptr(), 0 if q is None else _ld(q, q.shape, _FP8, "q"), None if s is None else s.data_ptr(),
                 None if qc is None else qc.data_ptr(), 0 if qc is None else _ld(qc, qc.shape, _FP8, "q_cols"), None if sc is None else sc.data_ptr())
    _check(lib().hgemm_fp8_quantize(ctx._h, ctypes.byref(d), _stream(ctx, stream)), f"hgemm_fp8_quantize(blocks={blocks}, {rows}x{cols})")


def _source(x, rows):
    """(rows, cols, ld, row pointer's checks) of the quantised matrix: x, or the rows of x that `rows` names."""
    if x.dim() != 2:
        raise ValueError("x must be a matrix")
    ld = _ld(x, x.shape, _WIDE, "x")
    if rows is None:
        return x.shape[0], x.shape[1], ld
    if rows.dim() != 1:
        raise ValueError("rows must be a vector of row numbers")
    _dense(rows, rows.shape, torch.int32, "rows")
    return rows.shape[0], x.shape[1], ld


def _row_copy(q, s, R, C):
    _ld(q, (R, C), _FP8, "q")
    _dense(s, (R, _blocks(C)), torch.float32, "scales")


def _col_copy(q, s, R, C, groups):
    r = padded_rows(R, groups) if groups else R
    _ld(q, (r, C), _FP8, "q_cols")
    _dense(s, (_blocks(r), C), torch.float32, "scales_cols")


def _groups_of(offsets):
    if offsets is None:
        return 0
    if offsets.dim() != 1 or offsets.shape[0] < 2:
        raise ValueError("offsets must be a vector of groups + 1 numbers")
    _dense(offsets, offsets.shape, torch.int32, "offsets")
    return offsets.shape[0] - 1


def quantize_rows(ctx, x, q, scales, rows=None, pow2: bool = False, stream=None) -> None:
    """1 x 128 blocks of x (fp32, fp16 or bf16 matrix); rows: int32 row numbers, row r of the result is row rows[r] of x
    (a row of zeros for a number outside it)."""
    R, C, ld = _source(x, rows)
    _row_copy(q, scales, R, C)
    _quantize(ctx, ROWS, x, (R, C), ld, rows, x.shape[0], None, 0, pow2, (q, scales), None, stream)


def quantize_cols(ctx, x, q, scales, rows=None, offsets=None, pow2: bool = False, stream=None) -> None:
    """128 x 1 blocks of x; offsets: blocks and copy per group (see ``empty_cols``)."""
    R, C, ld = _source(x, rows)
    groups = _groups_of(offsets)
    _col_copy(q, scales, R, C, groups)
    _quantize(ctx, COLS, x, (R, C), ld, rows, x.shape[0], offsets, groups, pow2, None, (q, scales), stream)


def quantize_both(ctx, x, q, scales, q_cols, scales_cols, rows=None, offsets=None, pow2: bool = False, stream=None) -> None:
    """The row and the column copy in one pass over x."""
    R, C, ld = _source(x, rows)
    groups = _groups_of(offsets)
    _row_copy(q, scales, R, C)
    _col_copy(q_cols, scales_cols, R, C, groups)
    _quantize(ctx, ROWS | COLS, x, (R, C), ld, rows, x.shape[0], offsets, groups, pow2, (q, scales), (q_cols, scales_cols), stream)


def quantize_tiles(ctx, x, q, scales, pow2: bool = False, stream=None) -> None:
    """128 x 128 tiles of a weight (N, K) or of a stack of them (groups, N, K)."""
    if x.dim() not in (2, 3):
        raise ValueError("x must be a matrix or a stack of matrices")
    ld = _ld(x, x.shape, _WIDE, "x")
    _ld(q, x.shape, _FP8, "q")
    R, C = x.shape[-2:]
    _dense(scales, (*x.shape[:-2], _blocks(R), _blocks(C)), torch.float32, "scales")
    _quantize(ctx, TILES, x, (R, C), ld, None, 0, None, x.shape[0] if x.dim() == 3 else 1, pow2, (q, scales), None, stream)


# ---- products ------------------------------------------------------------------------------------

class Plan:
    """``hgemm_fp8_plan`` / ``hgemm_fp8_run``: one of a layer's three products.

    form "forward": run(x (M,K), row scales, w (N,K), tile scales, y (M,N)); "input_grad": run(dy (M,N), row scales, w, tile
    scales, dx (M,K)); "weight_grad": run(dy (M,N), column scales, x (M,K), column scales, dw (N,K)).  groups > 0: one
    weight per group -- w (groups,N,K), dw (groups,N,K), ``offsets`` with every run, the weight gradient's operands
    laid out per group.

    Each plan holds one of the context's 4095 status words until it is closed or dropped; a program keeps its plans."""

    def __init__(self, ctx, M: int, N: int, K: int, form: str = "forward", groups: int = 0, a_dtype=torch.float8_e4m3fn, b_dtype=torch.float8_e4m3fn,
                 out_dtype=torch.bfloat16):
        if form not in FORMS:
            raise ValueError(f"form must be one of {', '.join(FORMS)}")
        if a_dtype not in _FP8 or b_dtype not in _FP8 or out_dtype not in _WIDE:
            raise ValueError("operands are float8_e4m3fn or float8_e5m2, results float32, float16 or bfloat16")
        self.ctx = ctx
        self.shape = (int(M), int(N), int(K))
        self.form, self.groups = form, int(groups)
        self._h = ctypes.c_void_p()
        self._run, self._destroy = lib().hgemm_fp8_run, lib().hgemm_fp8_plan_destroy
        _check(lib().hgemm_fp8_plan(ctx._h, FORMS[form], *self.shape, self.groups, TYPES[a_dtype], TYPES[b_dtype], TYPES[out_dtype], ctypes.byref(self._h)),
               f"hgemm_fp8_plan({form},{M},{N},{K},groups={groups})")
        M, N, K = self.shape
        g = (self.groups,) if self.groups else ()
        if form == "weight_grad":
            rows = padded_rows(M, self.groups) if self.groups else M
            a, sa, b, sb, c = (rows, N), (_blocks(rows), N), (rows, K), (_blocks(rows), K), (*g, N, K)
        else:
            a, c = ((M, K), (M, N)) if form == "forward" else ((M, N), (M, K))
            sa, b, sb = (M, _blocks(a[1])), (*g, N, K), (*g, _blocks(N), _blocks(K))
        self._a, self._sa, self._b, self._sb, self._c = (torch.Size(v) for v in (a, sa, b, sb, c))
        self._types = ((a_dtype,), (b_dtype,), (out_dtype,))

    @property
    def config(self) -> Config:
        c = Config()
        _check(lib().hgemm_fp8_plan_get_config(self._open(), ctypes.byref(c)), "hgemm_fp8_plan_get_config")
        return c

    def set_config(self, cta_group: int, block_q: int, split_k: int = 1) -> None:
        c = Config(cta_group, block_q, split_k, 0)
        _check(lib().hgemm_fp8_plan_set_config(self._open(), ctypes.byref(c)), f"hgemm_fp8_plan_set_config({c.as_dict()})")

    def _open(self):
        """The library's handle; none once the plan or its context is closed (the library then refuses the call)."""
        return self._h if self.ctx._h else None

    def last_device_status(self) -> tuple[int, int]:
        """``hgemm_fp8_last_device_status``: (status, code) of this plan's own status word; synchronises the device."""
        code = ctypes.c_uint32(0)
        st = lib().hgemm_fp8_last_device_status(self._open(), ctypes.byref(code))
        return int(st), int(code.value)

    def debug_timeout_probe(self, stream: int = 0) -> None:
        _check(lib().hgemm_fp8_debug_timeout_probe(self._open(), ctypes.c_void_p(stream)), "hgemm_fp8_debug_timeout_probe")

    def run(self, a, a_scales, b, b_scales, out, offsets=None, accumulate: bool = False, stream=None) -> None:
        ta, tb, tc = self._types
        lda, ldb, ldc = _ld(a, self._a, ta, "a"), _ld(b, self._b, tb, "b"), _ld(out, self._c, tc, "out")
        sa, sb = _dense(a_scales, self._sa, torch.float32, "a_scales"), _dense(b_scales, self._sb, torch.float32, "b_scales")
        off = None
        if self.groups:
            if offsets is None:
                raise ValueError("a plan with groups needs their offsets")
            off = _dense(offsets, (self.groups + 1,), torch.int32, "offsets")
        elif offsets is not None:
            raise ValueError("offsets belong to a plan with groups")
        st = self._run(self._open(), a.data_ptr(), lda, sa, b.data_ptr(), ldb, sb, out.data_ptr(), ldc, off, 1 if accumulate else 0, _stream(self.ctx, stream))
        if st != OK:
            raise HgemmError(st, f"hgemm_fp8_run({self.form}{self.shape}, groups={self.groups})")

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

"""The 4-bit products with block scales and their quantiser on the GPU, against plain forms.

Bytes that nothing may read hold patterns that would show (rows' ends, rows of other groups: the value 6 with scales of NaN), results sit inside
guard bands; the quantiser is checked bit for bit, products by bounds that follow from the arithmetic (fp4_reference.product_bound) or exactly."""
import ctypes
import subprocess
import zlib

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import fp4_reference as ref  # noqa: E402
from paper_2512_02551_b200 import build, fp4, hgemm  # noqa: E402

OUTS = [torch.float32, torch.float16, torch.bfloat16]
FORMATS = ["nvfp4", "mxfp4"]
CONFIGS = [(2, 256, 1), (2, 128, 1)] + [(1, bq, s) for bq in (64, 128) for s in (1, 2, 4, 8)]


@pytest.fixture(scope="module")
def ctx():
    assert torch.cuda.is_available(), "these tests need a B200"
    with hgemm.Context(0) as c:
        yield c


def rng(*key):
    return np.random.default_rng(zlib.crc32(repr(key).encode()))


def on_gpu(a, pitch_extra=0, fill=0xFF):
    """Bytes (..., R, n) as a view of a wider buffer whose other bytes are `fill`."""
    n = a.shape[-1]
    pitch = -(-n // 16) * 16 + pitch_extra
    wide = np.full((*a.shape[:-1], pitch), fill, np.uint8)
    wide[..., :n] = a
    return torch.from_numpy(wide).cuda()[..., :n]


class Operand:
    """Random codes and moderate scales of `shape`; places: the scale row of each row.  Scales that no row has are NaN (`spare`)."""

    def __init__(self, r, shape, fmt, places=None, scale_rows=None, integers=False, extra=16):
        *lead, R, C = shape
        B = ref.blocks(C, fmt)
        code = r.integers(0, 16, shape).astype(np.uint8)
        if integers:
            code = np.array([0, 2, 4, 10, 12], np.uint8)[r.integers(0, 5, shape)]             # 0, 1, 2, -1, -2
        lo, hi = ((0x28, 0x50) if fmt == "nvfp4" else (122, 132))
        s = r.integers(lo, hi, (*lead, R, B)).astype(np.uint8)
        if integers:
            s[:] = 0x38 if fmt == "nvfp4" else 127                                            # 1
        self.factor = None
        factor = np.ones(lead[0] if lead else 1)
        if fmt == "nvfp4":
            factor = np.exp2(r.integers(-3, 4, factor.shape)).astype(np.float32) * np.float32(1.0 if integers else 1.25)
            self.factor = torch.from_numpy(factor.astype(np.float32)).cuda()
        placed = s
        if places is not None:
            placed = np.full((scale_rows, B), 0x7F if fmt == "nvfp4" else 0xFF, np.uint8)
            placed[places] = s
        self.tiles = torch.from_numpy(ref.tiles_from(placed, fmt)).cuda()
        self.q = on_gpu(ref.pack(code), extra, 0x77)
        self.values = ref.decode(code) * ref.spread(ref.scale_values(s, fmt), fmt, C) * (factor.reshape(-1, 1, 1) if lead else factor[0])


def guarded(shape, dtype, offset=0, extra=0):
    """A result inside NaN: `extra` more elements per row, `offset` elements into its buffer."""
    rows, cols = int(np.prod(shape[:-1])), shape[-1]
    ld = cols + extra
    buf = torch.full((offset + rows * ld + 64,), float("nan"), dtype=dtype, device="cuda")
    out = buf[offset:offset + rows * ld].view(rows, ld)
    return buf, out[:, :cols] if len(shape) == 2 else out.view(*shape[:-1], ld)[..., :cols]


def untouched(buf, out):
    keep = torch.ones_like(buf, dtype=torch.bool)
    keep.as_strided(out.shape, out.stride(), out.storage_offset()).fill_(False)
    assert bool(torch.isnan(buf[keep]).all()), "something outside the result was written"


def shapes_of(form, M, N, K):
    """(A, B, result) of a form, both operands with the contraction last."""
    return {"forward": ((M, K), (N, K), (M, N)), "input_grad": ((M, N), (K, N), (M, K)), "weight_grad": ((N, M), (K, M), (N, K))}[form]


def dense_case(ctx, form, M, N, K, out_dtype, fmt="nvfp4", config=None, offset=0, extra=0, accumulate=False):
    r = rng(form, M, N, K, str(out_dtype), fmt)
    sa, sb, sc = shapes_of(form, M, N, K)
    a, b = Operand(r, sa, fmt), Operand(r, sb, fmt)
    buf, out = guarded(sc, out_dtype, offset, extra)
    before = None
    if accumulate:
        out.copy_(torch.from_numpy(r.standard_normal(sc)))
        before = ref.f64(out)
    with fp4.Plan(ctx, M, N, K, form=form, format=fmt, out_dtype=out_dtype) as plan:
        if config is not None:
            plan.set_config(*config)
        plan.run(a.q, a.tiles, b.q, b.tiles, out, a_factor=a.factor, b_factor=b.factor, accumulate=accumulate)
        st, code = plan.last_device_status()
        assert st == hgemm.OK, hex(code)
        untouched(buf, out)
        ref.check_product(out, a.values, b.values, f"{form} {M}x{N}x{K} {fmt} {out_dtype} {plan.config.as_dict()}", before)


SHAPES = [(1, 1, 1), (1, 128, 128), (3, 130, 257), (17, 64, 1000), (64, 300, 128), (129, 257, 385), (300, 520, 1040), (256, 256, 127)]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("config", CONFIGS, ids=str)
def test_every_kernel_at_small_and_odd_sizes(ctx, fmt, M, N, K, config):
    dense_case(ctx, "forward", M, N, K, OUTS[(M + N + K) % 3], fmt, config=config)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("form", ["input_grad", "weight_grad"])
@pytest.mark.parametrize("config", [(2, 256, 1), (1, 128, 1), (1, 64, 4)], ids=str)
def test_gradients(ctx, fmt, form, config):
    for i, (M, N, K) in enumerate([(1, 64, 64), (127, 1, 1), (130, 257, 100), (700, 300, 520)]):
        dense_case(ctx, form, M, N, K, OUTS[i % 3], fmt, config=config)


@pytest.mark.parametrize("config", [(2, 256, 1), (2, 128, 1), (1, 128, 1), (1, 64, 2)], ids=str)
@pytest.mark.parametrize("offset,extra", [(0, 0), (1, 0), (0, 3), (8, 8), (3, 5)])
def test_result_types_strides_and_alignment(ctx, config, offset, extra):
    for out_dtype in OUTS:
        for N in (200, 264):
            dense_case(ctx, "forward", 150, N, 190, out_dtype, config=config, offset=offset, extra=extra)


@pytest.mark.parametrize("form", ["forward", "weight_grad"])
@pytest.mark.parametrize("config", [(2, 256, 1), (2, 128, 1), (1, 128, 1), (1, 64, 4)], ids=str)
def test_accumulate(ctx, form, config):
    dense_case(ctx, form, 260, 300, 390, torch.float32, config=config, accumulate=True)


@pytest.mark.parametrize("fmt", FORMATS)
def test_several_waves_of_tiles(ctx, fmt):
    """More tiles than CTAs: every role walks on to further tiles, the accumulators change places; exact integers, so one misplaced element shows."""
    M, N, K = 2900, 3100, 2700
    r = rng(fmt)
    a, b = Operand(r, (M, K), fmt, integers=True), Operand(r, (N, K), fmt, integers=True)
    want = torch.from_numpy(a.values).cuda() @ torch.from_numpy(b.values).cuda().t()
    for out_dtype in (torch.float32, torch.bfloat16):
        for config in ((2, 256, 1), (2, 128, 1), (1, 128, 1), (1, 64, 1)):
            buf, out = guarded((M, N), out_dtype)
            with fp4.Plan(ctx, M, N, K, format=fmt, out_dtype=out_dtype) as plan:
                plan.set_config(*config)
                plan.run(a.q, a.tiles, b.q, b.tiles, out, a_factor=a.factor, b_factor=b.factor)
                assert plan.last_device_status()[0] == hgemm.OK
            untouched(buf, out)
            assert torch.equal(out, want.to(out_dtype)), (config, out_dtype)


@pytest.mark.parametrize("config", [(2, 256, 1), (2, 128, 1), (1, 64, 1), (1, 128, 4)], ids=str)
@pytest.mark.parametrize("fa,fb,small", [(-80, -80, False), (-99, -40, False), (-40, -99, False), (70, 60, True), (60, 70, True), (125, -126, False)])
def test_factors_whose_product_leaves_fp32(ctx, config, fa, fb, small):
    """Results are numbers where the product of the factors alone is none; rows of zeros stay zeros."""
    M, N, K = 140, 200, 390
    r = rng(config, fa, fb)
    a, b = Operand(r, (M, K), "nvfp4", integers=True), Operand(r, (N, K), "nvfp4", integers=True)
    scale = 1 if small else 0x7E                                    # 2^-9, or 448
    values = []
    for o, rows, e in ((a, M, fa), (b, N, fb)):
        code = np.where(r.random((rows, 1)) < 0.1, 0, r.integers(0, 16, (rows, K))).astype(np.uint8)
        o.q = on_gpu(ref.pack(code), 16, 0x77)
        o.tiles = torch.from_numpy(ref.tiles_from(np.full((rows, ref.blocks(K, "nvfp4")), scale, np.uint8), "nvfp4")).cuda()
        factor = np.float32(1.1) * np.float32(2.0) ** np.float32(e)
        o.factor = torch.tensor([factor], device="cuda")
        values.append(ref.decode(code) * ref.E4M3[scale] * float(factor))
    for out_dtype in (torch.float32, torch.bfloat16):
        buf, out = guarded((M, N), out_dtype)
        with fp4.Plan(ctx, M, N, K, out_dtype=out_dtype) as plan:
            plan.set_config(*config)
            plan.run(a.q, a.tiles, b.q, b.tiles, out, a_factor=a.factor, b_factor=b.factor)
            assert plan.last_device_status()[0] == hgemm.OK
        untouched(buf, out)
        ref.check_product(out, *values, f"{config} 2^{fa} 2^{fb}")
        assert bool((out != 0).any())


def test_launches_in_a_row_and_at_once(ctx):
    """Launches that follow one another without a pause, and two streams at once: the same bits each time."""
    M, N, K = 70, 500, 640
    r = rng(5)
    a, b = Operand(r, (M, K), "nvfp4"), Operand(r, (N, K), "nvfp4")
    for config in ((1, 64, 1), (1, 64, 8), (2, 256, 1), (2, 128, 1)):
        with fp4.Plan(ctx, M, N, K, out_dtype=torch.float32) as plan:
            plan.set_config(*config)
            outs = [torch.full((M, N), float("nan"), device="cuda") for _ in range(40)]
            streams = [torch.cuda.Stream() for _ in range(2)]
            torch.cuda.synchronize()
            for i, o in enumerate(outs):
                with torch.cuda.stream(streams[i % 2]):
                    plan.run(a.q, a.tiles, b.q, b.tiles, o, a_factor=a.factor, b_factor=b.factor)
            assert plan.last_device_status()[0] == hgemm.OK
            ref.check_product(outs[0], a.values, b.values, str(config))
            for o in outs[1:]:
                assert torch.equal(o, outs[0])


def test_nan_scales_stay_in_their_rows(ctx):
    """A block whose scale is NaN makes its row's results NaN, and no others."""
    for fmt in FORMATS:
        r = rng(fmt, 9)
        a, b = Operand(r, (200, 300), fmt), Operand(r, (140, 300), fmt)
        s = ref.scale_bytes(a.tiles, 200, 300, fmt).copy()
        s[7, 2] = s[150, 0] = 0x7F if fmt == "nvfp4" else 0xFF
        tiles = torch.from_numpy(ref.tiles_from(s, fmt)).cuda()
        for config in CONFIGS[::3]:
            out = torch.zeros(200, 140, device="cuda")
            with fp4.Plan(ctx, 200, 140, 300, format=fmt, out_dtype=torch.float32) as plan:
                plan.set_config(*config)
                plan.run(a.q, tiles, b.q, b.tiles, out, a_factor=a.factor, b_factor=b.factor)
            bad = torch.isnan(out).all(1)
            assert bad.nonzero().flatten().tolist() == [7, 150] and not torch.isnan(out[~bad]).any(), config


def test_no_rows(ctx):
    for form in ("forward", "input_grad", "weight_grad"):
        for groups in (0, 3):
            N, K = 64, 96
            plan = fp4.Plan(ctx, 0, N, K, form=form, groups=groups, out_dtype=torch.float32)
            a, b = (torch.zeros(*plan._a[:-1], -(-plan._a[-1] // 16) * 16, dtype=torch.uint8, device="cuda")[..., :plan._a[-1]],
                    torch.zeros(*plan._b[:-1], -(-plan._b[-1] // 16) * 16, dtype=torch.uint8, device="cuda")[..., :plan._b[-1]])
            sa, sb = torch.zeros(plan._sa, dtype=torch.uint8, device="cuda"), torch.zeros(plan._sb, dtype=torch.uint8, device="cuda")
            out = torch.full(tuple(plan._c), float("nan"), device="cuda")
            plan.run(a, sa, b, sb, out, a_factor=torch.ones(1, device="cuda"), b_factor=torch.ones(plan._b_factors, device="cuda"),
                     offsets=torch.zeros(groups + 1, dtype=torch.int32, device="cuda") if groups else None)
            torch.cuda.synchronize()
            assert form != "weight_grad" or bool((out == 0).all())
            plan.close()


# ---- products over experts ---------------------------------------------------------------------------

COUNTS = {
    "one of each": [1, 1, 1, 1],
    "empty ones": [0, 5, 0, 0, 130, 0],
    "one has all": [0, 0, 300, 0],
    "ragged": [128, 127, 129, 1, 0, 256, 255, 257, 16, 17, 65, 63],
    "many": [(7 * i) % 23 for i in range(70)],
    "all empty": [0, 0, 0],
}


def clamped(offsets, M):
    return np.maximum.accumulate(np.clip(offsets, 0, M))


def starts_of(offsets):
    """Where each group's rows begin if each begins at a multiple of 128."""
    padded = (np.diff(offsets) + 127) // 128 * 128
    return np.concatenate([[0], np.cumsum(padded)[:-1]])


def grouped_case(ctx, form, offsets, M, N, K, config, fmt="nvfp4", out_dtype=torch.float32, spoilt=None):
    """offsets: as they count; spoilt: what is handed over instead (falling or outside [0, M])."""
    E = len(offsets) - 1
    r = rng(form, E, M, N, K, fmt)
    start, counts = starts_of(offsets), np.diff(offsets)
    group = np.searchsorted(offsets, np.arange(M), side="right") - 1
    held = (group >= 0) & (group < E)
    room = fp4.padded_rows(M, E)
    places = np.where(held, start[np.clip(group, 0, E - 1)] + np.arange(M) - offsets[np.clip(group, 0, E - 1)], -1)
    off = torch.tensor(offsets if spoilt is None else spoilt, dtype=torch.int32, device="cuda")
    if form == "weight_grad":
        # columns outside the groups hold 6 with scales of NaN; a group's own padding holds zeros with scales of zero
        a, b = Operand(r, (N, room), fmt), Operand(r, (K, room), fmt)
        for o in (a, b):
            c, s = ref.codes(o.q, room).copy(), ref.scale_bytes(o.tiles, o.q.shape[0], room, fmt).copy()
            own, pad = np.zeros(room, bool), np.zeros(room, bool)
            for g in range(E):
                own[start[g]:start[g] + counts[g]] = True
                pad[start[g] + counts[g]:start[g] + (counts[g] + 127) // 128 * 128] = True
            nb = ref.BLOCK[fmt]
            c[:, pad], c[:, ~own & ~pad] = 0, 7
            s[:, ~(own | pad).reshape(-1, nb).any(1)] = 0x7F if fmt == "nvfp4" else 0xFF
            s[:, ~own.reshape(-1, nb).any(1) & pad.reshape(-1, nb).any(1)] = 0
            o.q, o.tiles = on_gpu(ref.pack(c), 16), torch.from_numpy(ref.tiles_from(s, fmt)).cuda()
            o.values = ref.decode(c) * ref.spread(ref.scale_values(s, fmt), fmt, room) * (1.0 if o.factor is None else float(o.factor))
        shape = (E, N, K)
    else:
        sa, sb, shape = shapes_of(form, M, N, K)
        a = Operand(r, sa, fmt, places[held], room) if held.all() else None
        if a is None:
            full = Operand(r, sa, fmt)
            s = np.full((room, ref.blocks(sa[1], fmt)), 0x7F if fmt == "nvfp4" else 0xFF, np.uint8)
            s[places[held]] = ref.scale_bytes(full.tiles, M, sa[1], fmt)[held]
            full.tiles = torch.from_numpy(ref.tiles_from(s, fmt)).cuda()
            a = full
        b = Operand(r, (E, *sb), fmt)
    buf, out = guarded(shape, out_dtype)
    with fp4.Plan(ctx, M, N, K, form=form, groups=E, format=fmt, out_dtype=out_dtype) as plan:
        if config is not None:
            plan.set_config(*config)
        plan.run(a.q, a.tiles, b.q, b.tiles, out, a_factor=a.factor, b_factor=b.factor, offsets=off)
        st, code = plan.last_device_status()
        assert st == hgemm.OK, hex(code)
        what = f"{form} {counts.tolist()} {plan.config.as_dict()} {fmt}"
    untouched(buf, out)
    for g in range(E):
        if form == "weight_grad":
            at = slice(start[g], start[g] + counts[g])
            ref.check_product(out[g], a.values[:, at], b.values[:, at], what + f" group {g}")
        elif counts[g]:
            at = slice(offsets[g], offsets[g + 1])
            ref.check_product(out[at], a.values[at], b.values[g], what + f" group {g}")
    if form != "weight_grad":
        assert bool(torch.isnan(out[torch.from_numpy(~held).cuda()]).all()), "rows of no group were written"


@pytest.mark.parametrize("form", ["forward", "input_grad", "weight_grad"])
@pytest.mark.parametrize("counts", COUNTS, ids=str)
@pytest.mark.parametrize("config", [(2, 256, 1), (2, 128, 1), (1, 64, 1), (1, 128, 1), (1, 64, 2)], ids=str)
def test_products_over_experts(ctx, form, counts, config):
    c = COUNTS[counts]
    if form == "weight_grad" and config[2] > 1 and len(c) > 20:
        config = (1, 128, 1)
    offsets = np.concatenate([[0], np.cumsum(c)])
    M = max(int(offsets[-1]), 5)
    grouped_case(ctx, form, offsets, M, 200, 264, config, FORMATS[(len(c) + config[1]) % 2], OUTS[len(c) % 3])


@pytest.mark.parametrize("form", ["forward", "weight_grad"])
def test_experts_planned_with_rows_of_no_group(ctx, form):
    grouped_case(ctx, form, np.array([0, 100, 230, 230, 500]), 700, 136, 320, None)
    grouped_case(ctx, form, np.array([0, 3, 4, 9, 9, 12, 30]), 30, 520, 520, None, "mxfp4", torch.bfloat16)


@pytest.mark.parametrize("form", ["forward", "weight_grad"])
@pytest.mark.parametrize("config", [(2, 256, 1), (1, 64, 1)], ids=str)
def test_offsets_that_fall_or_leave_the_rows(ctx, form, config):
    spoilt = np.array([0, 50, 30, 400, 350, 900])
    grouped_case(ctx, form, clamped(spoilt, 600), 600, 136, 200, config, spoilt=spoilt)


# ---- quantiser ---------------------------------------------------------------------------------------

def source(r, rows, cols, dtype, odd=True):
    """Values over many magnitudes, with blocks of zeros, exact ties and, where `odd`, NaN and infinities."""
    x = r.standard_normal((rows, cols)) * np.exp2(r.integers(-6, 7, (rows, cols)))
    x = np.where(r.random((rows, cols)) < 0.3, np.round(x * 4) / 4, x)
    x[r.random((rows, cols)) < 0.1] = 0
    for i in range(0, rows, 5):
        x[i, (16 * i) % max(1, cols):(16 * i) % max(1, cols) + 64] = 0
    t = torch.from_numpy(x).to(dtype)
    if odd and rows * cols > 40:
        flat = t.view(-1)
        at = r.integers(0, rows * cols, 3)
        flat[at[0]], flat[at[1]], flat[at[2]] = float("nan"), float("inf"), float("-inf")
    return t


def check_copy(q, tiles, x, fmt, factor, places=None, what=""):
    """A copy (values q, scale tiles) of x (fp32 values, R x C) bit for bit; places: the scale row of each row."""
    want_c, want_s = ref.quantize(x, fmt, factor)
    R, C = x.shape
    got = ref.codes(q, C)
    some = want_c != 255
    assert np.array_equal(np.where(some, ref.decode(got), 0), np.where(some, ref.decode(np.where(some, want_c, 0)), 0)), what + ": values"
    if C % 2:
        assert not (ref.bytes_of(q)[..., -1] >> 4).any(), what + ": an odd row's last half byte"
    t = ref.bytes_of(tiles)
    if places is None:
        assert np.array_equal(t, ref.tiles_from(want_s, fmt)), what + ": scales"
    else:
        assert np.array_equal(ref.scale_bytes(tiles, tiles.shape[0] * 128, C, fmt)[places], want_s), what + ": scales"


def empty_copy(shape, scale_shape, fmt):
    """Values and scales full of a pattern, rows 16 bytes further apart than they need be."""
    n = -(-shape[-1] // 2)
    q = torch.full((*shape[:-1], -(-n // 16) * 16 + 16), 0xA5, dtype=torch.uint8, device="cuda")[..., :n]
    s = torch.full(fp4._scales_shape(scale_shape, fmt), 0xA5, dtype=torch.uint8, device="cuda")
    return q, s


def rest_untouched(q):
    wide = q.as_strided((*q.shape[:-1], q.stride(-2)), q.stride())
    assert bool((wide[..., q.shape[-1]:] == 0xA5).all()), "bytes between the rows were written"


QUANT_SHAPES = [(1, 1), (1, 16), (3, 33), (24, 4096), (127, 129), (128, 128), (129, 257), (300, 640), (512, 77)]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", OUTS, ids=str)
@pytest.mark.parametrize("rows,cols", QUANT_SHAPES)
def test_quantise(ctx, fmt, dtype, rows, cols):
    r = rng(fmt, str(dtype), rows, cols)
    x = source(r, rows, cols, dtype)
    x64 = ref.f64(x)
    factors = [ref.tensor_factor(x64), 0.0123] if fmt == "nvfp4" else [None]
    for i, factor in enumerate(factors):
        wide = torch.full((rows, cols + (0, 8, 3)[(rows + i) % 3]), float("nan"), dtype=dtype, device="cuda")
        wide[:, :cols] = x
        xs = wide[:, :cols]
        f = None if factor is None else torch.tensor([factor], dtype=torch.float32, device="cuda")
        both = empty_copy((rows, cols), (rows, cols), fmt), empty_copy((cols, rows), (cols, rows), fmt)
        alone = empty_copy((rows, cols), (rows, cols), fmt), empty_copy((cols, rows), (cols, rows), fmt)
        fp4.quantize_both(ctx, xs, *both[0], *both[1], factor=f, format=fmt)
        fp4.quantize_rows(ctx, xs, *alone[0], factor=f, format=fmt)
        fp4.quantize_cols(ctx, xs, *alone[1], factor=f, format=fmt)
        for name, (row, col) in (("both", both), ("alone", alone)):
            check_copy(*row, x64.astype(np.float32), fmt, factor, what=f"{name} rows")
            check_copy(*col, np.ascontiguousarray(x64.T).astype(np.float32), fmt, factor, what=f"{name} columns")
            rest_untouched(row[0]), rest_untouched(col[0])


@pytest.mark.parametrize("fmt", FORMATS)
def test_quantise_every_tie(ctx, fmt):
    """Every scale against values halfway between two 4-bit values, from inputs of few bits: none of them goes astray."""
    steps = ref.E4M3[8:127] if fmt == "nvfp4" else np.exp2(np.arange(-20, 20))
    ties = np.array([6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, -0.75, -1.25, -1.75, -2.5, -3.5, -5.0, 4.0])
    x = (steps[:, None] * ties).astype(np.float32)
    x = np.repeat(x, 2, 1) if fmt == "mxfp4" else x
    for dtype in (torch.float32, torch.bfloat16):
        t = torch.from_numpy(x).to(dtype)
        assert np.array_equal(ref.f64(t), x)
        f = torch.ones(1, device="cuda") if fmt == "nvfp4" else None
        q, s = empty_copy(x.shape, x.shape, fmt)
        fp4.quantize_rows(ctx, t.cuda(), q, s, factor=f, format=fmt)
        check_copy(q, s, x, fmt, 1.0)
        want = ref.decode(ref.nearest_code(np.tile(ties, 1) if fmt == "nvfp4" else np.repeat(ties, 2)))
        assert np.array_equal(ref.decode(ref.codes(q, x.shape[1])), np.broadcast_to(want, x.shape))


def test_quantise_extremes(ctx):
    """Zeros, the smallest and the largest numbers, factors of zero and below 2^-100, values that a small factor saturates."""
    big = torch.finfo(torch.float32).max
    x = torch.zeros(8, 64)
    x[1], x[2], x[3], x[4, 3], x[5], x[6, ::2] = 1e-42, 2.0 ** -126, big, big, -1.0, 448 * 6.0
    for fmt in FORMATS:
        for factor in ([0.0, 1e-31, 2.0 ** -100, 1.0, 2.0 ** 117] if fmt == "nvfp4" else [None]):
            f = None if factor is None else torch.tensor([factor], device="cuda")
            q, s = empty_copy((8, 64), (8, 64), fmt)
            fp4.quantize_rows(ctx, x.cuda(), q, s, factor=f, format=fmt)
            check_copy(q, s, x.numpy(), fmt, factor, what=f"{fmt} {factor}")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
@pytest.mark.parametrize("factor", [2.0 ** -100, 2.0 ** -60, 1.5 * 2.0 ** -80])
def test_quantise_far_beyond_the_factor(ctx, dtype, factor):
    """A factor kept from smaller values: quotients beyond fp32 are 6 with their own sign, and the small values of such a block what they are elsewhere."""
    r = rng(str(dtype), factor)
    big = r.choice([-1e38, -1e25, -1e12, 1e12, 1e25, 1e38, -float(torch.finfo(torch.bfloat16).max)], (150, 200))
    small = r.choice([-7.0, -6.0, -5.0, -2.5, -0.25, 0.0, 0.25, 0.75, 1.75, 3.5, 9.0], (150, 200)) * 448.0 * np.float32(factor)
    x = torch.from_numpy(np.where(r.random((150, 200)) < 0.5, big, small)).to(dtype)
    x64 = ref.f64(x)
    f = torch.tensor([factor], dtype=torch.float32, device="cuda")
    both = empty_copy((150, 200), (150, 200), "nvfp4"), empty_copy((200, 150), (200, 150), "nvfp4")
    fp4.quantize_both(ctx, x.cuda(), *both[0], *both[1], factor=f)
    check_copy(*both[0], x64.astype(np.float32), "nvfp4", factor, what="rows")
    check_copy(*both[1], np.ascontiguousarray(x64.T).astype(np.float32), "nvfp4", factor, what="columns")


UNPACK = """
#include "fp4_quantize_kernel.cuh"
template <class T>
__global__ void unpack(const T *in, uint32_t *out)
{
    constexpr int kBytes = static_cast<int>(sizeof(T));
    uint32_t d[4];
    hgemm_dev::unpack_e2m1(in[threadIdx.x], d);
    for (int i = 0; i < kBytes; ++i) out[kBytes * threadIdx.x + i] = d[i];
}
extern "C" int run(int bytes, const void *in, uint32_t *out)
{
    if (bytes == 1) unpack<<<1, 256>>>(static_cast<const uint8_t *>(in), out);
    else if (bytes == 2) unpack<<<1, 256>>>(static_cast<const uint16_t *>(in), out);
    else unpack<<<1, 256>>>(static_cast<const uint32_t *>(in), out);
    return cudaDeviceSynchronize();
}
"""


def test_unpacking_words_of_which_a_part_is_known(tmp_path):
    """Codes to values from loads of 8, 16 and 32 bits, as many values as were loaded: what the compiler knows about the rest of a word changes nothing."""
    src, lib = tmp_path / "unpack.cu", tmp_path / "unpack.so"
    src.write_text(UNPACK)
    subprocess.run([build._nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-std=c++17", "-shared", "-Xcompiler", "-fPIC", "-I", build.CSRC, "-o", str(lib), str(src)], check=True)
    fn = ctypes.CDLL(str(lib)).run
    fn.argtypes = [ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p]
    for n, dtype in ((1, np.uint8), (2, np.uint16), (4, np.uint32)):
        words = rng("unpack", n).integers(0, 1 << (8 * n), 256).astype(dtype)
        code = np.stack([(words.astype(np.uint64) >> np.uint64(4 * i)) & np.uint64(15) for i in range(2 * n)], -1).astype(np.uint8)
        out = torch.empty(256, 2 * n, dtype=torch.float16, device="cuda")
        given = torch.from_numpy(words.view(np.uint8).copy()).cuda()
        assert fn(n, given.data_ptr(), out.data_ptr()) == 0
        assert np.array_equal(ref.f64(out), ref.decode(code)), n


@pytest.mark.parametrize("dtype", OUTS, ids=str)
def test_tensor_factor(ctx, dtype):
    for rows, cols, n in ((1, 1, 1), (7, 77, 1), (24, 4096, 1), (300, 128, 5), (1500, 1000, 1), (2048, 512, 3)):
        r = rng(rows, cols, n, str(dtype))
        x = torch.stack([source(r, rows, cols, dtype) * 2.0 ** -i for i in range(n)])
        for pad in (0, 3):
            wide = torch.full((n, rows, cols + pad), 1e4, dtype=dtype, device="cuda")
            wide[..., :cols] = x
            f = torch.full((n,), float("nan"), device="cuda")
            fp4.tensor_factor(ctx, wide[..., :cols] if n > 1 else wide[0, :, :cols], f)
            assert f.tolist() == [ref.tensor_factor(ref.f64(x[i])) for i in range(n)]
    for v in (0.0, float("nan"), float("inf")):
        f = torch.full((1,), 5.0, device="cuda")
        fp4.tensor_factor(ctx, torch.full((3, 40), v, dtype=dtype, device="cuda"), f)
        assert f.item() == 0.0
    f = torch.full((1,), 5.0, device="cuda")
    fp4.tensor_factor(ctx, torch.empty(0, 40, dtype=dtype, device="cuda"), f)
    assert f.item() == 0.0


@pytest.mark.parametrize("fmt", FORMATS)
def test_quantise_gathered_rows(ctx, fmt):
    r = rng(fmt)
    x = source(r, 50, 200, torch.bfloat16, odd=False)
    rows = r.integers(-3, 60, 333)
    rows[5], rows[6] = -(1 << 31), (1 << 31) - 1
    picked = np.where(((rows >= 0) & (rows < 50))[:, None], ref.f64(x)[np.clip(rows, 0, 49)], 0.0).astype(np.float32)
    f = torch.tensor([0.25], device="cuda") if fmt == "nvfp4" else None
    row, col = empty_copy((333, 200), (333, 200), fmt), empty_copy((200, 333), (200, 333), fmt)
    fp4.quantize_both(ctx, x.cuda(), *row, *col, factor=f, format=fmt, rows=torch.tensor(rows, dtype=torch.int32, device="cuda"))
    check_copy(*row, picked, fmt, 0.25)
    check_copy(*col, np.ascontiguousarray(picked.T), fmt, 0.25)
    # no rows to gather from: rows of zeros
    fp4.quantize_rows(ctx, torch.empty(0, 200, dtype=torch.bfloat16, device="cuda"), *row, factor=f, format=fmt, rows=torch.zeros(333, dtype=torch.int32, device="cuda"))
    check_copy(*row, np.zeros((333, 200), np.float32), fmt, 0.25)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16], ids=str)
@pytest.mark.parametrize("offsets", [[0, 0, 5, 5, 135, 400], [3, 50, 300, 400, 390], [0, 50, 30, 350, 300, 900], [0] + [40 * (i // 5 + 1) for i in range(45)], [0, 0, 0]], ids=str)
def test_quantise_per_group(ctx, fmt, dtype, offsets):
    M, C, E = 400, 200, len(offsets) - 1
    r = rng(fmt, E)
    x = source(r, M, C, dtype)
    x32 = ref.f64(x).astype(np.float32)
    off = clamped(np.array(offsets), M)
    start, room = starts_of(off), fp4.padded_rows(M, E)
    f, factor = (torch.tensor([0.5], device="cuda"), 0.5) if fmt == "nvfp4" else (None, None)
    given = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    for both in (True, False):
        row, col = empty_copy((M, C), (room, C), fmt), empty_copy((C, room), (C, room), fmt)
        if both:
            fp4.quantize_both(ctx, x.cuda(), *row, *col, factor=f, format=fmt, offsets=given)
        else:
            fp4.quantize_rows(ctx, x.cuda(), *row, factor=f, format=fmt, offsets=given)
            fp4.quantize_cols(ctx, x.cuda(), *col, factor=f, format=fmt, offsets=given)
        got_rows, got_cols = ref.bytes_of(row[0]), ref.bytes_of(col[0])
        end = 0
        for g in range(E):
            n = off[g + 1] - off[g]
            if not n:
                continue
            part, padded = x32[off[g]:off[g + 1]], (n + 127) // 128 * 128
            end = start[g] + padded
            tiles = slice(start[g] // 128, end // 128)
            check_copy(row[0][off[g]:off[g + 1]], row[1][tiles], part, fmt, factor, what=f"rows of group {g}")
            wide = np.zeros((C, padded), np.float32)
            wide[:, :n] = part.T
            atoms = 4 * ref.BLOCK[fmt]
            check_copy(col[0][:, start[g] // 2:end // 2], col[1][:, start[g] // atoms:end // atoms], wide, fmt, factor, what=f"columns of group {g}")
        assert (got_rows[:off[0]] == 0xA5).all() and (got_rows[off[-1]:] == 0xA5).all(), "rows of no group"
        assert (got_cols[:, end // 2:] == 0xA5).all(), "behind the last group"
        rest_untouched(row[0]), rest_untouched(col[0])
        # and back: a row copy with scale tiles per group
        if int(off[-1]) > 0:
            out = torch.full((M, C), 7.0, device="cuda")
            fp4.dequantize(ctx, *row, out, factor=f, format=fmt, offsets=given)
            places = np.concatenate([start[g] + np.arange(off[g + 1] - off[g]) for g in range(E)]).astype(np.int64)
            mine = slice(int(off[0]), int(off[-1]))
            want = ref.values(row[0][mine], row[1], C, fmt, 0.5 if factor else 1.0, places)
            assert np.array_equal(ref.f64(out)[mine], want, equal_nan=True)
            assert bool((out[:mine.start] == 7).all()) and bool((out[mine.stop:] == 7).all())


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("E", [64, 65, 100])
def test_quantise_many_groups_of_wide_rows(ctx, fmt, E):
    """More column tiles than CTAs share a row tile: with many groups each walks on to further ones."""
    M, C = 1300, 2700
    r = rng(fmt, E, "many")
    x = source(r, M, C, torch.bfloat16, odd=False)
    x32 = ref.f64(x).astype(np.float32)
    off = np.concatenate([[0], np.sort(r.integers(0, M + 1, E - 1)), [M]])
    start, room = starts_of(off), fp4.padded_rows(M, E)
    f, factor = (torch.tensor([0.5], device="cuda"), 0.5) if fmt == "nvfp4" else (None, None)
    given = torch.tensor(off, dtype=torch.int32, device="cuda")
    row, col = empty_copy((M, C), (room, C), fmt), empty_copy((C, room), (C, room), fmt)
    fp4.quantize_both(ctx, x.cuda(), *row, *col, factor=f, format=fmt, offsets=given)
    atoms = 4 * ref.BLOCK[fmt]
    for g in range(E):
        n = off[g + 1] - off[g]
        if n:
            end = start[g] + (n + 127) // 128 * 128
            check_copy(row[0][off[g]:off[g + 1]], row[1][start[g] // 128:end // 128], x32[off[g]:off[g + 1]], fmt, factor, what=f"rows of group {g}")
            wide = np.zeros((C, end - start[g]), np.float32)
            wide[:, :n] = x32[off[g]:off[g + 1]].T
            check_copy(col[0][:, start[g] // 2:end // 2], col[1][:, start[g] // atoms:end // atoms], wide, fmt, factor, what=f"columns of group {g}")
    out = torch.empty(M, C, device="cuda")
    fp4.dequantize(ctx, *row, out, factor=f, format=fmt, offsets=given)
    places = np.concatenate([start[g] + np.arange(off[g + 1] - off[g]) for g in range(E)])
    assert np.array_equal(ref.f64(out), ref.values(row[0], row[1], C, fmt, 0.5 if factor else 1.0, places))


@pytest.mark.parametrize("fmt", FORMATS)
def test_stacks(ctx, fmt):
    """A stack of weights: each matrix with its own factor; copies, and back."""
    G, R, C = 5, 130, 72
    r = rng(fmt, 1)
    x = torch.stack([source(r, R, C, torch.float32, odd=False) * 2.0 ** i for i in range(G)])
    f = None
    factors = [None] * G
    if fmt == "nvfp4":
        f = torch.empty(G, device="cuda")
        fp4.tensor_factor(ctx, x.cuda(), f)
        factors = f.tolist()
    row, col = empty_copy((G, R, C), (G, R, C), fmt), empty_copy((G, C, R), (G, C, R), fmt)
    fp4.quantize_both(ctx, x.cuda(), *row, *col, factor=f, format=fmt)
    back = torch.empty(G, R, C, device="cuda")
    fp4.dequantize(ctx, *row, back, factor=f, format=fmt)
    for i in range(G):
        x32 = ref.f64(x[i]).astype(np.float32)
        check_copy(row[0][i], row[1][i], x32, fmt, factors[i])
        check_copy(col[0][i], col[1][i], np.ascontiguousarray(x32.T), fmt, factors[i])
        assert np.array_equal(ref.f64(back[i]), ref.values(row[0][i], row[1][i], C, fmt, factors[i] or 1.0))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", OUTS, ids=str)
def test_dequantise(ctx, fmt, dtype):
    """Every code and every scale, odd sizes, strides, alignments."""
    for i, (R, C) in enumerate(((1, 1), (256, 64), (130, 333), (7, 4096))):
        r = rng(fmt, R, C)
        code, s = r.integers(0, 16, (R, C)).astype(np.uint8), r.integers(0, 127 if fmt == "nvfp4" else 256, (R, ref.blocks(C, fmt))).astype(np.uint8)
        factor = 0.3 if fmt == "nvfp4" else None
        buf, out = guarded((R, C), dtype, (0, 1, 8)[i % 3], (0, 3, 8, 5)[i])
        f = None if factor is None else torch.tensor([factor], device="cuda")
        fp4.dequantize(ctx, on_gpu(ref.pack(code)), torch.from_numpy(ref.tiles_from(s, fmt)).cuda(), out, factor=f, format=fmt)
        if fmt == "nvfp4":
            v = ref.decode(code).astype(np.float32) * ref.spread((ref.E4M3[s].astype(np.float32) * np.float32(factor)), fmt, C)
        else:
            with np.errstate(over="ignore"):
                v = ref.decode(code) * ref.spread(ref.scale_values(s, fmt), fmt, C)
        want = torch.from_numpy(v.astype(np.float64)).float().to(dtype)
        assert torch.equal(torch.nan_to_num(out.cpu(), nan=12345.0), torch.nan_to_num(want, nan=12345.0))
        torch.cuda.synchronize()
        keep = torch.ones_like(buf, dtype=torch.bool)
        keep.as_strided(out.shape, out.stride(), out.storage_offset()).fill_(False)
        assert bool(torch.isnan(buf[keep]).all())


def test_quantise_a_large_matrix(ctx):
    """More tiles than fit the GPU at once; some of its rows and columns."""
    x = torch.randn(8191, 2050, device="cuda", dtype=torch.bfloat16)
    f = torch.empty(1, device="cuda")
    fp4.tensor_factor(ctx, x, f)
    row, col = empty_copy((8191, 2050), (8191, 2050), "nvfp4"), empty_copy((2050, 8191), (2050, 8191), "nvfp4")
    fp4.quantize_both(ctx, x, *row, *col, factor=f)
    for at in (0, 4096, 8064):
        check_copy(row[0][at:at + 128], row[1][at // 128:at // 128 + 1], ref.f64(x[at:at + 128]).astype(np.float32), "nvfp4", f.item())
    part = ref.f64(x[:, :128].t().contiguous()).astype(np.float32)
    check_copy(col[0][:128], col[1][:1], part, "nvfp4", f.item())


# ---- together ----------------------------------------------------------------------------------------

@pytest.mark.parametrize("fmt", FORMATS)
def test_a_layers_step_and_its_gradients(ctx, fmt):
    """Quantiser and products as a training step uses them; the gradients against the formula's on the dequantised operands, and against differences of
    the layer that those operands define."""
    M, N, K = 200, 136, 264
    g = torch.Generator(device="cuda").manual_seed(4)
    x, w, dy = (torch.randn(*s, generator=g, device="cuda") for s in ((M, K), (N, K), (M, N)))
    held = {}

    def copies(t, name):
        f = None
        if fmt == "nvfp4":
            f = torch.empty(1, device="cuda")
            fp4.tensor_factor(ctx, t, f)
        rows, cols = fp4.empty_rows(*t.shape, format=fmt), fp4.empty_cols(*t.shape, format=fmt)
        fp4.quantize_both(ctx, t, *rows, *cols, factor=f, format=fmt)
        held[name] = rows, cols, f
        back = torch.empty_like(t), torch.empty(t.shape[1], t.shape[0], device="cuda")
        fp4.dequantize(ctx, *rows, back[0], factor=f, format=fmt)
        fp4.dequantize(ctx, *cols, back[1], factor=f, format=fmt)
        return back[0].double(), back[1].double()

    (x_r, x_c), (w_r, w_c), (dy_r, dy_c) = copies(x, "x"), copies(w, "w"), copies(dy, "dy")
    assert (x_r - x.double()).norm() < 0.15 * x.double().norm() and (x_c.t() - x.double()).norm() < 0.15 * x.double().norm()
    out = {f: torch.empty(s, device="cuda") for f, s in (("forward", (M, N)), ("input_grad", (M, K)), ("weight_grad", (N, K)))}
    pick = {"forward": ("x", 0, "w", 0), "input_grad": ("dy", 0, "w", 1), "weight_grad": ("dy", 1, "x", 1)}
    for form, (a, i, b, j) in pick.items():
        with fp4.Plan(ctx, M, N, K, form=form, format=fmt, out_dtype=torch.float32) as plan:
            plan.run(*held[a][i], *held[b][j], out[form], a_factor=held[a][2], b_factor=held[b][2])
            assert plan.last_device_status()[0] == hgemm.OK
    # a sum of n products in 32 bits is off by at most n 2^-23 of its magnitudes
    for form, (p, q) in {"forward": (x_r, w_r), "input_grad": (dy_r, w_c), "weight_grad": (dy_c, x_c)}.items():
        bound = (p.shape[1] + 5) * 2.0 ** -23 * (p.abs() @ q.abs().t()) + 2.0 ** -150
        assert bool(((out[form].double() - p @ q.t()).abs() <= bound).all()), form
    # differences: L(x) = sum(dy * x w^T) with the copies that each gradient reads; L is linear, so that any step gives the slope
    v = torch.randn(M, K, generator=g, device="cuda").double()
    slope = (dy_r * ((x_r + v) @ w_c)).sum() - (dy_r * (x_r @ w_c)).sum()
    assert abs(float((out["input_grad"].double() * v).sum() - slope)) < 1e-4 * float((dy_r.abs() * (v.abs() @ w_c.abs())).sum())
    u = torch.randn(N, K, generator=g, device="cuda").double()
    slope = (dy_c.t() * (x_c.t() @ (w_r + u).t())).sum() - (dy_c.t() * (x_c.t() @ w_r.t())).sum()
    assert abs(float((out["weight_grad"].double() * u).sum() - slope)) < 1e-4 * float((dy_c.t().abs() * (x_c.t().abs() @ u.abs().t())).sum())


def test_captured_and_replayed(ctx):
    """Factor, quantiser and product in one graph, replayed on new inputs."""
    M, N, K = 33, 256, 512
    w = torch.randn(N, K, device="cuda")
    wf, xf = torch.empty(1, device="cuda"), torch.empty(1, device="cuda")
    wq, xq = fp4.empty_rows(N, K), fp4.empty_rows(M, K)
    fp4.tensor_factor(ctx, w, wf)
    fp4.quantize_rows(ctx, w, *wq, factor=wf)
    x, y = torch.zeros(M, K, device="cuda", dtype=torch.bfloat16), torch.empty(M, N, device="cuda")
    plan = fp4.Plan(ctx, M, N, K, out_dtype=torch.float32)

    def step():
        fp4.tensor_factor(ctx, x, xf)
        fp4.quantize_rows(ctx, x, *xq, factor=xf)
        plan.run(*xq, *wq, y, a_factor=xf, b_factor=wf)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(3):
        x.copy_(torch.randn(M, K, device="cuda") * 10.0 ** i)
        graph.replay()
        got = y.clone()
        step()
        assert torch.equal(got, y) and float(y.abs().max()) > 0
    plan.close()


def test_large_stacks_of_weights(ctx):
    """A stack of weights of more than 2^32 values, its last matrices used: offsets pass 32 bits."""
    E, N, K = 520, 2048, 4096
    q, s = torch.zeros(E, N, K // 2, dtype=torch.uint8, device="cuda"), torch.zeros(E, N // 128, K // 64, 512, dtype=torch.uint8, device="cuda")
    r = rng(77)
    w = Operand(r, (N, K), "nvfp4", extra=0)
    for e in (511, 519):
        q[e], s[e] = w.q, w.tiles
    M = 40
    offsets = np.zeros(E + 1, np.int64)
    offsets[512:] = 25
    offsets[520:] = 40
    start = starts_of(offsets)
    places = np.concatenate([start[511] + np.arange(25), start[519] + np.arange(15)])
    a = Operand(r, (M, K), "nvfp4", places, fp4.padded_rows(M, E))
    out = torch.full((M, N), float("nan"), device="cuda")
    with fp4.Plan(ctx, M, N, K, groups=E, out_dtype=torch.float32) as plan:
        for config in (None, (2, 256, 1)):
            if config:
                plan.set_config(*config)
            plan.run(a.q, a.tiles, q, s, out, a_factor=a.factor, b_factor=w.factor.expand(E).contiguous(), offsets=torch.tensor(offsets, dtype=torch.int32, device="cuda"))
            assert plan.last_device_status()[0] == hgemm.OK
            ref.check_product(out, a.values, w.values)


def test_large_results(ctx):
    """Results of more than 2^31 elements: a matrix, and a stack of gradients whose last ones have rows."""
    M, N, K = 70000, 40008, 64
    r = rng("large result")
    a, b = Operand(r, (M, K), "nvfp4"), Operand(r, (N, K), "nvfp4")
    out = torch.full((M, N), float("nan"), dtype=torch.bfloat16, device="cuda")
    at = np.concatenate([np.arange(3), r.integers(0, M, 20), np.arange(M - 40, M)])
    for config in ((2, 256, 1), (2, 128, 1), (1, 128, 1)):
        with fp4.Plan(ctx, M, N, K) as plan:
            plan.set_config(*config)
            plan.run(a.q, a.tiles, b.q, b.tiles, out, a_factor=a.factor, b_factor=b.factor)
            assert plan.last_device_status()[0] == hgemm.OK
        ref.check_product(out[torch.from_numpy(at).cuda()], a.values[at], b.values, str(config))
        assert not bool(torch.isnan(out).any())
        out.fill_(float("nan"))
    del out
    E, N, K = 600, 2000, 2056
    counts = np.zeros(E, np.int64)
    counts[[0, 1, 598, 599]] = 5, 130, 100, 70
    offsets = np.concatenate([[0], np.cumsum(counts)])
    M, start = int(offsets[-1]), starts_of(offsets)
    room = fp4.padded_rows(M, E)
    a, b = Operand(r, (N, room), "mxfp4"), Operand(r, (K, room), "mxfp4")
    own = np.zeros(room, bool)
    for e in np.flatnonzero(counts):
        own[start[e]:start[e] + counts[e]] = True
    for o in (a, b):                                               # columns of no row: zeros with scales of their own
        c = ref.codes(o.q, room).copy()
        c[:, ~own] = 0
        o.q, o.values = on_gpu(ref.pack(c), 16), o.values * own
    out = torch.full((E, N, K), float("nan"), dtype=torch.bfloat16, device="cuda")
    for config in ((2, 256, 1), (1, 64, 1)):
        with fp4.Plan(ctx, M, N, K, form="weight_grad", groups=E, format="mxfp4") as plan:
            plan.set_config(*config)
            plan.run(a.q, a.tiles, b.q, b.tiles, out, offsets=torch.tensor(offsets, dtype=torch.int32, device="cuda"))
            assert plan.last_device_status()[0] == hgemm.OK
        for e in (0, 1, 598, 599):
            at = slice(start[e], start[e] + counts[e])
            ref.check_product(out[e], a.values[:, at], b.values[:, at], f"{config} {e}")
        assert float(out[2:598].abs().max()) == 0
        out.fill_(float("nan"))


@pytest.mark.parametrize("fmt", FORMATS)
def test_quantise_beyond_32_bits(ctx, fmt):
    """A matrix of more than 2^31 elements, both ways; its corners."""
    R, C = 66000, 33000
    g = torch.Generator(device="cuda").manual_seed(9)
    x = torch.randn(R, C, dtype=torch.bfloat16, generator=g, device="cuda")
    f = torch.full((1,), 2.0 ** -8, device="cuda") if fmt == "nvfp4" else None
    factor = 2.0 ** -8 if fmt == "nvfp4" else None
    row, col = fp4.empty_rows(R, C, format=fmt), fp4.empty_cols(R, C, format=fmt)
    fp4.quantize_both(ctx, x, *row, *col, factor=f, format=fmt)
    top, left = R // 128 * 128, C // 128 * 128                      # where the last tiles begin
    check_copy(row[0][top:], row[1][top // 128:], ref.f64(x[top:]).astype(np.float32), fmt, factor)
    check_copy(col[0][left:], col[1][left // 128:], ref.f64(x[:, left:].t().contiguous()).astype(np.float32), fmt, factor)
    back = torch.empty_like(x)
    fp4.dequantize(ctx, *row, back, factor=f, format=fmt)
    want = ref.values(row[0][top:], row[1][top // 128:], C, fmt, 1.0 if factor is None else factor)
    assert np.array_equal(ref.f64(back[top:]), ref.f64(torch.from_numpy(want).bfloat16()))
    if f is not None:
        x[-1, -1] = 3000.0
        fp4.tensor_factor(ctx, x, f)
        assert f.item() == 2.0


# ---- refusals ----------------------------------------------------------------------------------------

def test_refusals(ctx):
    L, bad = fp4.lib(), hgemm.ERR_INVALID_ARG
    x = torch.zeros(64, 64, device="cuda")
    q, s = fp4.empty_rows(64, 64)
    f = torch.ones(1, device="cuda")
    good = dict(blocks=1, x_type=0, format=0, matrices=1, rows=64, cols=64, ldx=64, x=x.data_ptr(), row_index=None, x_rows=64, offsets=None, groups=0, reserved=0, factor=f.data_ptr(),
                q=q.data_ptr(), ldq=32, scales=s.data_ptr(), q_cols=q.data_ptr(), ldq_cols=32, scales_cols=s.data_ptr())
    call = lambda **kw: L.hgemm_fp4_quantize(ctx._h, ctypes.byref(fp4.Quantize(**{**good, **kw})), None)  # noqa: E731
    assert call() == hgemm.OK
    for kw in (dict(blocks=0), dict(blocks=4), dict(x_type=3), dict(format=2), dict(matrices=0), dict(matrices=1025), dict(rows=-1), dict(cols=0), dict(ldx=63), dict(x=None),
               dict(x=x.data_ptr() + 2), dict(q=None), dict(q=q.data_ptr() + 8), dict(ldq=24), dict(ldq=16), dict(scales=None), dict(scales=s.data_ptr() + 4), dict(factor=None),
               dict(format=1), dict(groups=1), dict(offsets=f.data_ptr()), dict(offsets=f.data_ptr() + 2, groups=1), dict(offsets=f.data_ptr(), groups=1025),
               dict(offsets=f.data_ptr(), groups=1, matrices=2), dict(row_index=f.data_ptr() + 1), dict(row_index=f.data_ptr(), x_rows=-1), dict(row_index=f.data_ptr(), matrices=2),
               dict(blocks=2, q_cols=None), dict(blocks=3, ldq_cols=16), dict(blocks=2, scales_cols=None), dict(rows=(1 << 22) + 1)):
        assert call(**kw) == bad, kw
    deq = lambda *a: L.hgemm_fp4_dequantize(ctx._h, *a, None)  # noqa: E731
    args = [0, 0, 1, 64, 64, q.data_ptr(), 32, s.data_ptr(), f.data_ptr(), None, 0, x.data_ptr(), 64]
    assert deq(*args) == hgemm.OK
    for i, v in ((0, 2), (1, 3), (2, 0), (3, -1), (4, 0), (5, None), (5, q.data_ptr() + 1), (6, 16), (6, 40), (7, None), (8, None), (10, 1), (11, None), (11, x.data_ptr() + 1), (12, 63)):
        assert deq(*[v if j == i else a for j, a in enumerate(args)]) == bad, (i, v)
    fac = [0, 1, 64, 64, x.data_ptr(), 64, f.data_ptr(), None]
    assert L.hgemm_fp4_tensor_factor(ctx._h, *fac) == hgemm.OK
    for i, v in ((0, 3), (1, 0), (2, -1), (3, 0), (4, None), (5, 63), (6, None)):
        assert L.hgemm_fp4_tensor_factor(ctx._h, *[v if j == i else a for j, a in enumerate(fac)]) == bad, (i, v)
    with fp4.Plan(ctx, 64, 64, 64, out_dtype=torch.bfloat16) as plan:
        out = torch.zeros(64, 64, dtype=torch.bfloat16, device="cuda")
        run = [q.data_ptr(), 32, s.data_ptr(), f.data_ptr(), q.data_ptr(), 32, s.data_ptr(), f.data_ptr(), out.data_ptr(), 64, None, 0]
        go = lambda a: L.hgemm_fp4_run(plan._h, *a, None)  # noqa: E731
        assert go(run) == hgemm.OK
        for i, v in ((0, None), (0, q.data_ptr() + 8), (1, 16), (1, 40), (2, None), (2, s.data_ptr() + 8), (3, None), (4, None), (5, 24), (6, None), (7, None), (8, None), (8, out.data_ptr() + 1),
                     (9, 63), (10, f.data_ptr()), (11, 1), (11, 2)):
            assert go([v if j == i else a for j, a in enumerate(run)]) == bad, (i, v)
        with pytest.raises(ValueError):
            plan.run(q, s, q, s, out)                                         # no factors
        with pytest.raises(ValueError):
            plan.run(q, s, q, s, out, a_factor=f, b_factor=f, offsets=torch.zeros(2, dtype=torch.int32, device="cuda"))
        with pytest.raises(ValueError):
            plan.run(q[:32], s, q, s, out, a_factor=f, b_factor=f)
        for c in ((2, 64, 1), (2, 256, 2), (1, 32, 1), (1, 256, 1), (1, 64, 3), (3, 64, 1)):
            with pytest.raises(hgemm.HgemmError):
                plan.set_config(*c)
        plan.debug_timeout_probe()
        assert plan.last_device_status()[0] != hgemm.OK and plan.last_device_status()[0] == hgemm.OK
    with pytest.raises(hgemm.HgemmError):
        fp4.Plan(ctx, 1, 0, 1)
    with pytest.raises(hgemm.HgemmError):
        fp4.Plan(ctx, 1, 1, 1, groups=1025)


def test_a_closed_plan_and_context_refuse():
    c = hgemm.Context(0)
    plan = fp4.Plan(c, 8, 64, 64)
    q, s = fp4.empty_rows(8, 64)
    w, ws = fp4.empty_rows(64, 64)
    f, out = torch.ones(1, device="cuda"), torch.zeros(8, 64, dtype=torch.bfloat16, device="cuda")
    plan.close()
    with pytest.raises(hgemm.HgemmError):
        plan.run(q, s, w, ws, out, a_factor=f, b_factor=f)
    plan = fp4.Plan(c, 8, 64, 64)
    c.close()
    with pytest.raises(hgemm.HgemmError):
        plan.run(q, s, w, ws, out, a_factor=f, b_factor=f)

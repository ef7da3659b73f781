"""The 8-bit products with block scales and their quantiser on the GPU, against plain 64-bit forms.

Inputs hold NaN wherever nothing may be read (columns between a matrix's width and its row distance, rows of other groups) and
results sit inside guard bands; the tolerances follow from the arithmetic (fp8_reference.product_bound)."""
import zlib

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import fp8_reference as ref  # noqa: E402
from paper_2512_02551_b200 import fp8, hgemm  # noqa: E402

OUTS = [torch.float32, torch.float16, torch.bfloat16]
E4M3, E5M2 = torch.float8_e4m3fn, torch.float8_e5m2


@pytest.fixture(scope="module")
def ctx():
    assert torch.cuda.is_available(), "these tests need a B200"
    with hgemm.Context(0) as c:
        yield c


def rng(*key):
    return torch.Generator(device="cuda").manual_seed(zlib.crc32(repr(key).encode()))


def bytes8(g, shape, dtype, spread=1.0):
    """8-bit values over most of the type's range, rows 16 bytes (or more) apart, NaN between them."""
    pitch = -(-shape[-1] // 16) * 16 + 16
    wide = torch.full((*shape[:-1], pitch), 0x7F, dtype=torch.uint8, device="cuda").view(dtype)
    v = (torch.randn(*shape, generator=g, device="cuda") * spread * 20.0).clamp(-400, 400).to(dtype)
    wide.view(torch.uint8)[..., :shape[-1]] = v.view(torch.uint8)
    return wide[..., :shape[-1]]


def scales(g, *shape):
    return torch.rand(*shape, generator=g, device="cuda") * 0.01 + 1e-4


def guarded(shape, dtype, offset=0, extra=0):
    """A result inside NaN: `extra` more elements per row, `offset` elements into its buffer."""
    rows, cols = int(np.prod(shape[:-1])), shape[-1]
    ld = cols + extra
    buf = torch.full((offset + rows * ld + 64,), float("nan"), dtype=dtype, device="cuda")
    out = buf[offset:offset + rows * ld].view(rows, ld)
    return buf, out[:, :cols] if len(shape) == 2 else out.view(*shape[:-1], ld)[..., :cols]


def untouched(buf, out):
    """Nothing outside `out` was written, everything inside was."""
    assert not bool(torch.isnan(out).any()), "some element of the result was never written"
    n = out.numel()
    assert int(torch.isnan(buf).sum()) == buf.numel() - n, "the kernel wrote outside its result"


def blocks(n):
    return -(-n // 128)


def dense_case(ctx, form, M, N, K, out_dtype, a_dtype=E4M3, config=None, offset=0, extra=0, accumulate=False):
    g = rng(form, M, N, K, str(out_dtype))
    if form == "weight_grad":
        a, b = bytes8(g, (M, N), a_dtype), bytes8(g, (M, K), E4M3)
        sa, sb = scales(g, blocks(M), N), scales(g, blocks(M), K)
        p, q, nb, shape = ref.values(a, sa, 128, 1).T, ref.values(b, sb, 128, 1).T, blocks(M), (N, K)
    else:
        a, b = bytes8(g, (M, K) if form == "forward" else (M, N), a_dtype), bytes8(g, (N, K), E4M3)
        sa, sb = scales(g, M, blocks(a.shape[1])), scales(g, blocks(N), blocks(K))
        w = ref.values(b, sb, 128, 128)
        p, q, nb, shape = ref.values(a, sa, 1, 128), w if form == "forward" else w.T, blocks(a.shape[1]), (M, N) if form == "forward" else (M, K)
    buf, out = guarded(shape, out_dtype, offset, extra)
    if accumulate:
        out.copy_(torch.randn(*shape, generator=g, device="cuda"))
        before = ref.f64(out)
    with fp8.Plan(ctx, M, N, K, form=form, a_dtype=a_dtype, out_dtype=out_dtype) as plan:
        if config is not None:
            plan.set_config(*config)
        plan.run(a, sa, b, sb, out, accumulate=accumulate)
        st, code = ctx.last_device_status()
        assert st == hgemm.OK, hex(code)
        untouched(buf, out)
        if accumulate:
            exact = p @ q.T
            bound = ref.product_bound(np.abs(p) @ np.abs(q).T + np.abs(before), nb, out_dtype, exact + before)
            assert (np.abs(ref.f64(out) - exact - before) <= bound).all()
        else:
            ref.check_product(out, p, q, nb, f"{form} {M}x{N}x{K} {out_dtype} {plan.config.as_dict()}")


SWAPPED = [(1, bq, s) for bq in (16, 32, 64, 128) for s in (1, 2, 4, 8)]
SHAPES = [(1, 1, 1), (1, 128, 128), (3, 130, 257), (17, 64, 1000), (64, 300, 128), (129, 257, 384), (300, 520, 1040), (256, 256, 128)]


@pytest.mark.parametrize("form", ["forward", "input_grad"])
@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("config", [(2, 256, 1)] + SWAPPED, ids=str)
def test_every_kernel_at_small_and_odd_sizes(ctx, form, M, N, K, config):
    dense_case(ctx, form, M, N, K, OUTS[(M + N + K) % 3], config=config)


@pytest.mark.parametrize("M,N,K", [(1, 64, 64), (127, 1, 1), (128, 130, 257), (130, 256, 100), (1000, 129, 384), (700, 520, 300)])
@pytest.mark.parametrize("config", [(2, 256, 1), (1, 128, 1), (1, 128, 2), (1, 128, 4), (1, 128, 8)], ids=str)
def test_weight_gradient_kernels(ctx, M, N, K, config):
    dense_case(ctx, "weight_grad", M, N, K, OUTS[(M + N + K) % 3], config=config)


@pytest.mark.parametrize("form", ["forward", "input_grad", "weight_grad"])
@pytest.mark.parametrize("out_dtype", OUTS, ids=str)
@pytest.mark.parametrize("a_dtype", [E4M3, E5M2], ids=str)
def test_types(ctx, form, out_dtype, a_dtype):
    dense_case(ctx, form, 200, 384, 272, out_dtype, a_dtype=a_dtype)
    dense_case(ctx, form, 200, 384, 272, out_dtype, a_dtype=a_dtype, config=(2, 256, 1))


@pytest.mark.parametrize("form", ["forward", "input_grad", "weight_grad"])
@pytest.mark.parametrize("config", [(2, 256, 1), (1, 128, 1), (1, 128, 4)], ids=str)
@pytest.mark.parametrize("offset,extra", [(1, 0), (0, 3), (8, 8), (3, 5)])
def test_result_strides_and_alignment(ctx, form, config, offset, extra):
    for out_dtype in OUTS:
        dense_case(ctx, form, 150, 200, 190, out_dtype, config=config, offset=offset, extra=extra)


@pytest.mark.parametrize("form", ["forward", "input_grad", "weight_grad"])
@pytest.mark.parametrize("config", [(2, 256, 1), (1, 128, 1), (1, 128, 4)], ids=str)
def test_accumulate(ctx, form, config):
    dense_case(ctx, form, 260, 300, 390, torch.float32, config=config, accumulate=True)


@pytest.mark.parametrize("form", ["forward", "input_grad", "weight_grad"])
def test_several_waves_of_tiles(ctx, form):
    """More tiles than CTAs: every role walks on to further tiles; exact integers, so one misplaced element shows."""
    M, N, K = 2900, 3100, 2700
    g = rng(form)
    small = lambda r, c: torch.randint(-2, 3, (r, c), generator=g, device="cuda").float()  # noqa: E731
    ones = lambda *s: torch.full(s, 0.5, device="cuda")  # noqa: E731
    x = {"forward": (M, K), "input_grad": (M, N), "weight_grad": (M, N)}[form]
    w = (M, K) if form == "weight_grad" else (N, K)
    fa, fb = small(*x), small(*w)
    a, b = fp8.empty_rows(*x)[0], fp8.empty_rows(*w)[0]
    a.copy_(fa), b.copy_(fb)
    if form == "weight_grad":
        sa, sb, want = ones(blocks(M), N), ones(blocks(M), K), fa.double().t() @ fb.double()
    else:
        sa, sb = ones(M, blocks(x[1])), ones(blocks(N), blocks(K))
        want = fa.double() @ (fb.double().t() if form == "forward" else fb.double())
    for config in ((2, 256, 1), (1, 128, 1), (1, 128, 2)):
        buf, out = guarded(tuple(want.shape), torch.float32)
        with fp8.Plan(ctx, M, N, K, form=form, out_dtype=torch.float32) as plan:
            plan.set_config(*config)
            plan.run(a, sa, b, sb, out)
            assert ctx.last_device_status()[0] == hgemm.OK
        untouched(buf, out)
        assert torch.equal(out.double(), want * 0.25), config


def test_no_rows(ctx):
    for form in ("forward", "input_grad", "weight_grad"):
        for groups in (0, 3):
            g = (groups,) if groups else ()
            N, K = 64, 96
            shape = (*g, N, K) if form == "weight_grad" else (0, N if form == "forward" else K)
            rows = fp8.padded_rows(0, groups) if groups else 0
            a = torch.empty(rows if form == "weight_grad" else 0, K if form == "forward" else N, dtype=E4M3, device="cuda")
            b = torch.empty(*((rows, K) if form == "weight_grad" else (*g, N, K)), dtype=E4M3, device="cuda")
            sa = torch.empty(blocks(rows), N, device="cuda") if form == "weight_grad" else torch.empty(0, blocks(a.shape[1]), device="cuda")
            sb = torch.empty(blocks(rows), K, device="cuda") if form == "weight_grad" else torch.empty(*g, 1, 1, device="cuda")
            out = torch.full(shape, float("nan"), device="cuda")
            with fp8.Plan(ctx, 0, N, K, form=form, groups=groups, out_dtype=torch.float32) as plan:
                plan.run(a, sa, b, sb, out, offsets=torch.zeros(groups + 1, dtype=torch.int32, device="cuda") if groups else None)
            torch.cuda.synchronize()
            assert form != "weight_grad" or bool((out == 0).all())


# ---- products over experts ---------------------------------------------------------------------------

COUNTS = {
    "one of each": [1, 1, 1, 1],
    "empty ones": [0, 5, 0, 0, 130, 0],
    "one has all": [0, 0, 300, 0],
    "ragged": [128, 127, 129, 1, 0, 256, 255, 257, 16, 17],
    "many": [(7 * i) % 23 for i in range(70)],
    "all empty": [0, 0, 0],
}


def grouped_case(ctx, form, counts, N, K, config, out_dtype=torch.float32, spare=0):
    """`spare`: rows behind the last group, which belong to none."""
    E, M = len(counts), sum(counts) + spare
    if M == 0:
        M = spare = 5
    g = rng(form, E, M, N, K)
    offsets = torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32, device="cuda")
    ends = offsets.tolist()
    if form == "weight_grad":
        rows = fp8.padded_rows(M, E)
        a, b = bytes8(g, (rows, N), E4M3), bytes8(g, (rows, K), E4M3)
        sa, sb = scales(g, blocks(rows), N), scales(g, blocks(rows), K)
        at, held = 0, torch.zeros(rows, dtype=torch.bool, device="cuda")
        want = []
        for n in counts:
            held[at:at + n] = True
            up = blocks(n) * 128
            if n < up:
                a.view(torch.uint8)[at + n:at + up] = 0
                b.view(torch.uint8)[at + n:at + up] = 0
            want.append((at, n))
            at += up
        a.view(torch.uint8)[at:] = 0x7F                     # behind the last group: never read
        b.view(torch.uint8)[at:] = 0x7F
        pa, pb = ref.values(a, sa, 128, 1), ref.values(b, sb, 128, 1)
        pairs = [(pa[s:s + n].T, pb[s:s + n].T, blocks(n)) for s, n in want]
        shape = (E, N, K)
    else:
        a, w = bytes8(g, (M, K if form == "forward" else N), E4M3), bytes8(g, (E, N, K), E4M3)
        w = w.reshape(E, N, -1) if w.is_contiguous() else w
        sa, sb = scales(g, M, blocks(a.shape[1])), scales(g, E, blocks(N), blocks(K))
        va, vw = ref.values(a, sa, 1, 128), ref.values(w, sb, 128, 128)
        pairs = [(va[ends[e]:ends[e + 1]], vw[e] if form == "forward" else vw[e].T, blocks(a.shape[1])) for e in range(E)]
        b, shape = w, (M, N if form == "forward" else K)
    buf, out = guarded(shape, out_dtype)
    with fp8.Plan(ctx, M, N, K, form=form, groups=E, out_dtype=out_dtype) as plan:
        if config is not None:
            plan.set_config(*config)
        plan.run(a, sa, b, sb, out, offsets=offsets)
        assert ctx.last_device_status()[0] == hgemm.OK
        what = f"{form} {counts} {N}x{K} {plan.config.as_dict()}"
    if form == "weight_grad":
        untouched(buf, out)
    else:
        n = ends[-1]
        assert bool(torch.isnan(out[n:]).all()), "rows of no group were written"
        if n:
            assert not bool(torch.isnan(out[:n]).any()) and int(torch.isnan(buf).sum()) == buf.numel() - n * shape[1]
    for e, (p, q, nb) in enumerate(pairs):
        got = out[e] if form == "weight_grad" else out[ends[e]:ends[e + 1]]
        if got.numel():
            ref.check_product(got, p, q, nb, f"{what} group {e}")


@pytest.mark.parametrize("form", ["forward", "input_grad"])
@pytest.mark.parametrize("counts", list(COUNTS), ids=str)
@pytest.mark.parametrize("config", [None, (2, 256, 1), (1, 16, 1), (1, 32, 2), (1, 64, 1), (1, 128, 4)], ids=str)
def test_experts_rows(ctx, form, counts, config):
    grouped_case(ctx, form, COUNTS[counts], 272, 200, config, OUTS[len(counts) % 3], spare=3 if counts == "ragged" else 0)


@pytest.mark.parametrize("counts", list(COUNTS), ids=str)
@pytest.mark.parametrize("config", [None, (2, 256, 1), (1, 128, 1), (1, 128, 4)], ids=str)
def test_experts_weight_gradient(ctx, counts, config):
    grouped_case(ctx, "weight_grad", COUNTS[counts], 144, 272, config, OUTS[len(counts) % 3])


@pytest.mark.parametrize("form", ["forward", "input_grad", "weight_grad"])
@pytest.mark.parametrize("K", [1, 65, 100, 256])
def test_experts_of_one_output(ctx, form, K):
    """Weights of one row: stacks whose matrices are rows, of any width."""
    for out_dtype in OUTS:
        grouped_case(ctx, form, [3, 0, 130, 1], 1, K, None, out_dtype)


def test_experts_offsets_out_of_range_stay_inside(ctx):
    """Offsets beyond the rows, negative or falling are clamped: nothing outside the operands is touched."""
    M, N, K, E = 40, 64, 128, 4
    g = rng("offsets")
    a, w = bytes8(g, (M, K), E4M3), bytes8(g, (E, N, K), E4M3)
    sa, sb = scales(g, M, 1), scales(g, E, 1, 1)
    for bad in ([0, 10, 5, 2000000000, 50], [-5, -1, 20, 10, 40], [7, 7, 7, 7, 1 << 30]):
        for config in ((2, 256, 1), (1, 16, 1)):
            buf, out = guarded((M, N), torch.float32)
            with fp8.Plan(ctx, M, N, K, groups=E, out_dtype=torch.float32) as plan:
                plan.set_config(*config)
                plan.run(a, sa, w, sb, out, offsets=torch.tensor(bad, dtype=torch.int32, device="cuda"))
                assert ctx.last_device_status()[0] == hgemm.OK
            assert bool(torch.isnan(buf[M * N:]).all())


# ---- order of work ---------------------------------------------------------------------------------------

def test_streams_and_repeats_give_the_same_bits(ctx):
    """Two streams at once, and calls after one another with other operands between them: the same bits as alone."""
    M, N, K = 70, 512, 2048
    g = rng("streams")
    sets = []
    for _ in range(3):
        x, w = torch.randn(M, K, generator=g, device="cuda", dtype=torch.float32), torch.randn(N, K, generator=g, device="cuda")
        sets.append((x, w, *fp8.empty_rows(M, K), *fp8.empty_tiles(N, K)))
    plan = fp8.Plan(ctx, M, N, K, out_dtype=torch.float32)

    def chain(s, out, stream=None):
        x, w, q, sc, wq, ws = s
        fp8.quantize_rows(ctx, x, q, sc, stream=stream)
        fp8.quantize_tiles(ctx, w, wq, ws, stream=stream)
        plan.run(q, sc, wq, ws, out, stream=stream)

    alone = []
    for s in sets:
        out = torch.empty(M, N, device="cuda")
        chain(s, out)
        torch.cuda.synchronize()
        alone.append(out)
    streams = [torch.cuda.Stream() for _ in sets]
    outs = [torch.empty(M, N, device="cuda") for _ in sets]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, o, st in zip(sets, outs, streams):
            chain(s, o, st.cuda_stream)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(alone, outs))
    # captured into a graph
    graph, out = torch.cuda.CUDAGraph(), torch.empty(M, N, device="cuda")
    with torch.cuda.graph(graph):
        chain(sets[1], out)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, alone[1])
    plan.close()


def test_short_launches_one_after_another(ctx):
    """Tiles of one block, pairs and single CTAs in turn on the same SMs, with nothing between the launches: each CTA leaves while its last
    commits are recent.  Exact integers."""
    M, N, K = 1100, 1300, 128
    g = rng("short")
    fa, fb = (torch.randint(-2, 3, s, generator=g, device="cuda").float() for s in ((M, K), (N, K)))
    a, b = fp8.empty_rows(M, K)[0], fp8.empty_rows(N, K)[0]
    a.copy_(fa), b.copy_(fb)
    sa, sb = torch.full((M, 1), 0.5, device="cuda"), torch.full((blocks(N), 1), 0.5, device="cuda")
    want = fa @ fb.t() * 0.25
    plans = []
    for config in ((2, 256, 1), (1, 16, 1), (1, 128, 1)):
        plans.append(fp8.Plan(ctx, M, N, K, out_dtype=torch.float32))
        plans[-1].set_config(*config)
    outs = [torch.full((M, N), float("nan"), device="cuda") for _ in range(60)]
    for i, out in enumerate(outs):
        plans[i % 3].run(a, sa, b, sb, out)
    assert ctx.last_device_status()[0] == hgemm.OK
    assert all(torch.equal(out, want) for out in outs)
    for plan in plans:
        plan.close()


def test_status_words(ctx):
    """A wait that ran out is reported by the plan whose launch it was, by the context, and by the context too when the plan is gone
    before anyone asks."""
    one, two = fp8.Plan(ctx, 64, 64, 64), fp8.Plan(ctx, 64, 64, 64)
    ctx.set_wait_budget(2_000_000)                      # about a millisecond
    try:
        one.debug_timeout_probe()
        assert two.last_device_status() == (hgemm.OK, 0)
        st, code = one.last_device_status()
        assert st == hgemm.ERR_TIMEOUT and (code >> 24) == 4
        assert one.last_device_status() == (hgemm.OK, 0) and ctx.last_device_status() == (hgemm.OK, 0)
        two.debug_timeout_probe()
        assert ctx.last_device_status()[0] == hgemm.ERR_TIMEOUT and two.last_device_status() == (hgemm.OK, 0)
        two.debug_timeout_probe()
        two.close()
        st, code = ctx.last_device_status()
        assert st == hgemm.ERR_TIMEOUT and (code >> 24) == 4
        assert ctx.last_device_status() == (hgemm.OK, 0)
    finally:
        ctx.set_wait_budget(2_000_000_000)
    one.close()


def test_dropped_plans_give_their_place_back():
    """A context has room for 4095 plans at once; plans and layers that are dropped or closed make room for others."""
    from paper_2512_02551_b200.run_experts import ExpertLayer
    with hgemm.Context(0) as c:
        for i in range(5000):
            fp8.Plan(c, 1 + i % 100, 64, 64)
        held = [fp8.Plan(c, 1, 64, 64) for _ in range(4095 - 7)]
        for _ in range(2):
            with ExpertLayer(c, 8, 128, 128, 2, 1) as layer:              # seven plans
                layer.forward(torch.zeros(8, 128, dtype=torch.float16, device="cuda"))
                with pytest.raises(hgemm.HgemmError):
                    fp8.Plan(c, 1, 64, 64)
        assert c.last_device_status() == (hgemm.OK, 0)
        del held
        c.plan(256, 256, 256).close()


def test_plans_open_at_exit():
    """A program that ends with open plans ends without a word on stderr."""
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    code = "from paper_2512_02551_b200 import fp8, hgemm\nctx = hgemm.Context(0)\nplan = fp8.Plan(ctx, 16, 64, 128)\nkept = [fp8.Plan(ctx, 16, 64, 128)]\nprint('made')\n"
    out = subprocess.run([sys.executable, "-c", code], env=dict(os.environ, PYTHONPATH=root), capture_output=True, text=True, timeout=300)
    assert out.returncode == 0 and out.stdout == "made\n" and "Exception" not in out.stderr and "Error" not in out.stderr, out.stderr


# ---- quantisation --------------------------------------------------------------------------------------------

def check_quantized(q, s, x, rows, cols, name, pow2, what):
    """Scales within 2^-23 of the definition (powers of two exactly), values those of the definition, one code off only where the
    three roundings of the factor and the product (2^-23 each) reach across the middle between two codes."""
    v, want_s = ref.quantize(x, rows, cols, name, pow2)
    got_s = ref.f64(s)
    assert got_s.shape == want_s.shape
    assert (got_s == want_s).all() if pow2 else (np.abs(got_s - want_s) <= 2.0 ** -23 * want_s).all(), what
    got = ref.f64(q)
    assert (np.isnan(got) == np.isnan(v)).all(), what
    ok = ~np.isnan(v)
    lo, hi = ref.nearest(v[ok] * (1 - 3 * 2.0 ** -23), name), ref.nearest(v[ok] * (1 + 3 * 2.0 ** -23), name)
    near = (got[ok] == lo) | (got[ok] == hi)
    assert near.all(), f"{what}: {int((~near).sum())} of {near.size} values"


def awkward(g, R, C, dtype):
    x = torch.randn(R, C, generator=g, device="cuda") * torch.exp(2.0 * torch.randn(R, 1, generator=g, device="cuda"))
    x[::7, ::5] = 0.0
    if R > 4:
        x[3] = 0.0                                          # a row of zeros
        x[4, :] = 1e-8
        x[2, C // 2] = 60000.0
    if C > 140 and R > 2:
        x[1, 0:128] = 0.0
        x[1, 130], x[0, 5], x[2, 7] = float("nan"), float("inf"), -float("inf")
    return x.to(dtype)


QSHAPES = [(1, 1), (1, 128), (2, 129), (5, 1000), (128, 128), (130, 300), (257, 96), (300, 513)]


@pytest.mark.parametrize("R,C", QSHAPES)
@pytest.mark.parametrize("dtype", OUTS, ids=str)
@pytest.mark.parametrize("name", ["e4m3", "e5m2"])
@pytest.mark.parametrize("pow2", [False, True])
def test_quantize(ctx, R, C, dtype, name, pow2):
    x = awkward(rng(R, C, name), R, C, dtype)
    xs = ref.f64(x)
    f8 = ref.FP8[name]
    q, s = fp8.empty_rows(R, C, f8)
    fp8.quantize_rows(ctx, x, q, s, pow2=pow2)
    check_quantized(q, s, xs, 1, 128, name, pow2, "rows")
    t, st = fp8.empty_tiles(R, C, dtype=f8)
    fp8.quantize_tiles(ctx, x, t, st, pow2=pow2)
    check_quantized(t, st, xs, 128, 128, name, pow2, "tiles")
    c, sc = fp8.empty_cols(R, C, dtype=f8)
    fp8.quantize_cols(ctx, x, c, sc, pow2=pow2)
    check_quantized(c, sc, xs, 128, 1, name, pow2, "cols")
    q2, s2 = fp8.empty_rows(R, C, f8)
    c2, sc2 = fp8.empty_cols(R, C, dtype=f8)
    fp8.quantize_both(ctx, x, q2, s2, c2, sc2, pow2=pow2)
    for u, v in ((q, q2), (c, c2)):
        assert torch.equal(u.contiguous().view(torch.uint8), v.contiguous().view(torch.uint8))
    assert torch.equal(s, s2) and torch.equal(sc, sc2)


def test_quantize_extremes(ctx):
    x = torch.zeros(6, 256, device="cuda")
    x[0, 3] = 3.4e38
    x[1, 4] = 2.0 ** -100
    x[2, 5] = 2.0 ** -101
    x[3, :] = float("nan")
    x[4, :] = float("inf")
    x[5, 1], x[5, 2] = 1e-40, -0.0
    for pow2 in (False, True):
        for name in ("e4m3", "e5m2"):
            q, s = fp8.empty_rows(6, 256, ref.FP8[name])
            fp8.quantize_rows(ctx, x, q, s, pow2=pow2)
            check_quantized(q, s, ref.f64(x), 1, 128, name, pow2, "extremes")


def test_quantize_strides_and_guards(ctx):
    """x with any row distance and any base; the copy's own row distance; nothing written between the rows."""
    g = rng("strides")
    for dtype in OUTS:
        for R, C, extra, shift in ((9, 200, 1, 1), (130, 130, 7, 3), (64, 256, 8, 8)):
            base = torch.randn(R * (C + extra) + shift, generator=g, device="cuda").to(dtype)
            x = base[shift:].view(R, C + extra)[:, :C]
            wide = torch.full((R, 320), 0x55, dtype=torch.uint8, device="cuda")
            wide_c = wide.clone()
            q, c = wide.view(E4M3)[:, :C], wide_c.view(E4M3)[:, :C]
            s, sc = torch.empty(R, blocks(C), device="cuda"), torch.empty(blocks(R), C, device="cuda")
            fp8.quantize_both(ctx, x, q, s, c, sc)
            check_quantized(q, s, ref.f64(x), 1, 128, "e4m3", False, "rows")
            check_quantized(c, sc, ref.f64(x), 128, 1, "e4m3", False, "cols")
            assert bool((wide[:, C:] == 0x55).all()) and bool((wide_c[:, C:] == 0x55).all())


def test_quantize_gather_from_nothing(ctx):
    """A source without rows: every row number lies outside it, the copies are zeros with scales of 1."""
    x = torch.empty(0, 200, dtype=torch.bfloat16, device="cuda")
    rows = torch.arange(-2, 3, dtype=torch.int32, device="cuda")
    q, s = fp8.empty_rows(5, 200)
    c, t = fp8.empty_cols(5, 200)
    for v in (q, c):
        v.view(torch.uint8).fill_(0x7F)
    fp8.quantize_rows(ctx, x, q, s, rows)
    fp8.quantize_both(ctx, x, q, s, c, t, rows)
    for values, scale in ((q, s), (c, t)):
        assert bool((values.view(torch.uint8) == 0).all()) and bool((scale == 1).all())


def test_quantize_gather(ctx):
    g = rng("gather")
    x = torch.randn(50, 300, generator=g, device="cuda").to(torch.bfloat16)
    rows = torch.randint(0, 50, (333,), generator=g, device="cuda", dtype=torch.int32)
    rows[::9] = -1
    rows[5] = 50                                             # outside: rows of zeros
    picked = ref.f64(x)[np.clip(rows.cpu().numpy(), 0, 49)]
    picked[(rows.cpu().numpy() < 0) | (rows.cpu().numpy() > 49)] = 0.0
    q, s = fp8.empty_rows(333, 300)
    fp8.quantize_rows(ctx, x, q, s, rows=rows)
    check_quantized(q, s, picked, 1, 128, "e4m3", False, "gathered rows")
    c, sc = fp8.empty_cols(333, 300)
    fp8.quantize_cols(ctx, x, c, sc, rows=rows)
    check_quantized(c, sc, picked, 128, 1, "e4m3", False, "gathered columns")


@pytest.mark.parametrize("counts", list(COUNTS), ids=str)
def test_quantize_per_group(ctx, counts):
    counts = COUNTS[counts]
    E, M, C = len(counts), sum(counts) + 2, 200
    g = rng("groups", M)
    x = torch.randn(M, C, generator=g, device="cuda")
    offsets = torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32, device="cuda")
    q, s = fp8.empty_rows(M, C)
    c, sc = fp8.empty_cols(M, C, E)
    c.view(torch.uint8)[:] = 0x55
    sc.fill_(-1.0)
    fp8.quantize_both(ctx, x, q, s, c, sc, offsets=offsets)
    n = sum(counts)
    if n:
        check_quantized(q[:n], s[:n], ref.f64(x)[:n], 1, 128, "e4m3", False, "rows")
    c1, sc1 = fp8.empty_cols(M, C, E)
    fp8.quantize_cols(ctx, x, c1, sc1, offsets=offsets)
    at, start = 0, 0
    for n in counts:
        up = blocks(n) * 128
        if n:
            check_quantized(c[at:at + n], sc[at // 128:(at + up) // 128], ref.f64(x)[start:start + n], 128, 1, "e4m3", False, "a group's columns")
            assert bool((c[at + n:at + up].float() == 0).all())
            assert torch.equal(c[at:at + up].contiguous().view(torch.uint8), c1[at:at + up].contiguous().view(torch.uint8))
        at, start = at + up, start + n
    assert bool((c.view(torch.uint8)[at:] == 0x55).all()) and bool((sc[at // 128:] == -1.0).all())


def test_quantize_tiles_of_one_row(ctx):
    """Stacks of one-row matrices, dense or taken out of a larger stack."""
    g = rng("one row")
    for C in (1, 65, 128, 300):
        wide = torch.randn(4, 5, C, generator=g, device="cuda")
        for x in (torch.randn(4, 1, C, generator=g, device="cuda"), wide[:, 2:3], wide[1:2, 2:3]):
            q, s = fp8.empty_tiles(*x.shape)
            fp8.quantize_tiles(ctx, x, q, s)
            for e in range(x.shape[0]):
                check_quantized(q[e], s[e], ref.f64(x[e]), 128, 128, "e4m3", False, f"matrix {e} of {tuple(x.shape)}")
    with pytest.raises(ValueError):
        fp8.quantize_tiles(ctx, wide[:1, :1].expand(4, 1, 300), *fp8.empty_tiles(4, 1, 300))


def definition32(x, name, pow2, rows, cols):
    """Values and scales by the header's definition, every step one correctly rounded 32-bit operation (tensors divide tensors: a number as
    the divisor or the dividend becomes a product with a reciprocal)."""
    R, C = x.shape
    x = x.float()
    b = torch.nn.functional.pad(x, (0, -C % cols, 0, -R % rows)).view(blocks(R) if rows > 1 else R, rows, -(-C // cols), cols)
    amax = torch.where(torch.isfinite(b), b.abs(), 0.0).amax((1, 3), keepdim=True)
    some = amax >= 2.0 ** -100
    a, top = torch.where(some, amax, 1.0), torch.full_like(amax, ref.FP8_MAX[name])
    scale = a / top
    factor = top / a
    if pow2:
        mantissa, exponent = torch.frexp(scale)
        exponent = exponent - (mantissa == 0.5).int()
        scale, factor = torch.ldexp(torch.ones_like(scale), exponent), torch.ldexp(torch.ones_like(scale), -exponent)
    v = (b * torch.where(some, factor, 0.0)).clamp(-ref.FP8_MAX[name], ref.FP8_MAX[name])
    v = torch.where(torch.isfinite(b), v, torch.nan).to(ref.FP8[name])
    bits = v.view(torch.uint8).reshape(-(-R // rows) * rows, -(-C // cols) * cols)[:R, :C]
    return bits, torch.where(some, scale, 1.0)[:, 0, :, 0]


def same_as_definition(q, s, x, name, pow2, rows, cols, what):
    bits, scale = definition32(x, name, pow2, rows, cols)
    got = q.view(torch.uint8)
    nan = torch.isnan(q.float())
    assert torch.equal(nan, ~torch.isfinite(x.float())), what
    off = (got != bits) & ~nan
    assert not bool(off.any()), f"{what}: {int(off.sum())} of {off.numel()} values, first at {off.nonzero()[0].tolist()}"
    assert torch.equal(s, scale), what


@pytest.mark.parametrize("dtype", OUTS, ids=str)
@pytest.mark.parametrize("name", ["e4m3", "e5m2"])
@pytest.mark.parametrize("pow2", [False, True])
def test_quantize_bit_for_bit(ctx, dtype, name, pow2):
    """All forms against the definition in 32 bits: the same bits."""
    for R, C in ((24, 4096), (700, 520)):
        x = awkward(rng("bits", R, C), R, C, dtype)
        q, s = fp8.empty_rows(R, C, ref.FP8[name])
        c, sc = fp8.empty_cols(R, C, dtype=ref.FP8[name])
        fp8.quantize_both(ctx, x, q, s, c, sc, pow2=pow2)
        same_as_definition(q, s, x, name, pow2, 1, 128, "rows with columns")
        same_as_definition(c, sc, x, name, pow2, 128, 1, "columns")
        fp8.quantize_rows(ctx, x, q, s, pow2=pow2)
        same_as_definition(q, s, x, name, pow2, 1, 128, "rows")
        t, st = fp8.empty_tiles(R, C, dtype=ref.FP8[name])
        fp8.quantize_tiles(ctx, x, t, st, pow2=pow2)
        same_as_definition(t, st, x, name, pow2, 128, 128, "tiles")


# rows, columns, extra elements between rows, shift of the base, gathered: each with more blocks than the threshold from which a lane
# has four of them in flight (1024 a multiprocessor: 151552)
MANY = {
    "dense, last group partly filled": (50523, 384, 0, 0, False),
    "dense, long rows": (1187, 16384, 0, 0, False),
    "groups straddle rows": (19001, 1000, 0, 0, False),
    "more than a group a row, ragged": (7601, 2469, 3, 0, False),
    "unaligned": (7601, 2469, 0, 1, False),
    "whole rows apart": (8000, 2432, 8, 8, False),
    "one block a row": (151777, 100, 4, 0, False),
    "gathered": (7601, 2469, 3, 0, True),
    "gathered whole blocks": (9500, 2048, 0, 0, True),
}


@pytest.mark.parametrize("case", list(MANY), ids=str)
@pytest.mark.parametrize("dtype", OUTS, ids=str)
@pytest.mark.parametrize("name", ["e4m3", "e5m2"])
def test_quantize_many_rows(ctx, case, dtype, name):
    """The row kernels for large inputs, with NaN and infinities in first and last blocks of a warp's sixteen, bit for bit."""
    R, C, extra, shift, gathered = MANY[case]
    g = rng("many", case)
    source = R // 2 if gathered else R
    base = (torch.randn(source * (C + extra) + shift, generator=g, device="cuda") * 3.0).to(dtype)
    x = base[shift:].view(source, C + extra)[:, :C]
    per_row = blocks(C)
    for b, at, value in ((0, 0, float("inf")), (15, 5, float("nan")), (16, 99, -float("inf")), (31, 64, float("inf")), (source * per_row // 2, 1, float("nan")),
                         (source * per_row - 1, 7, float("inf")), (source * per_row - 17, 3, -float("inf"))):
        r, k = divmod(b, per_row)
        x[r, min(k * 128 + at, C - 1)] = value
    x[source // 3] = 0.0
    rows, want = None, x
    if gathered:
        rows = torch.randint(0, source, (R,), generator=g, device="cuda", dtype=torch.int32)
        rows[:3], rows[-1], rows[100::977] = torch.tensor([0, -1, source]), source - 1, source + 5
        inside = (rows >= 0) & (rows < source)
        want = torch.where(inside.unsqueeze(1), x[rows.clamp(0, source - 1).long()], torch.zeros((), dtype=dtype, device="cuda"))
    q, s = fp8.empty_rows(R, C, ref.FP8[name])
    assert R * per_row >= 1024 * torch.cuda.get_device_properties(0).multi_processor_count
    fp8.quantize_rows(ctx, x, q, s, rows=rows)
    same_as_definition(q, s, want, name, False, 1, 128, case)


FALLING = {
    "falls and overshoots": (40, [0, 10, 5, 2000000000, 50]),
    "negative": (40, [-5, -1, 20, 10, 40]),
    "starts late": (40, [7, 7, 7, 7, 1 << 30]),
    "up and down": (1000, [0, 1000] * 4 + [0]),
    "up and down, many": (300, [0, 300, -1, 150] * 25 + [299]),
    "falls between chunks of 32": (500, list(range(0, 32)) + [400, 3] + list(range(4, 40)) + [450]),
}


@pytest.mark.parametrize("case", list(FALLING), ids=str)
@pytest.mark.parametrize("both", [False, True], ids=["cols", "both"])
def test_quantize_offsets_out_of_range_stay_inside(ctx, case, both):
    """Offsets that are negative, fall or reach beyond the rows count as the products count them -- clamped to the rows, each at least
    as large as those before it -- and nothing behind the padded copy or its scales is written."""
    M, bad = FALLING[case]
    C, E, spare = 200, len(bad) - 1, 100                      # spare: blocks behind the copy
    x = torch.randn(M, C, generator=rng("falling", case), device="cuda")
    capacity = fp8.padded_rows(M, E)
    wide = torch.full((capacity + spare * 128, 208), 0x55, dtype=torch.uint8, device="cuda")
    wide_s = torch.full((blocks(capacity) + spare, C), -1.0, device="cuda")
    c, sc = wide[:capacity, :C].view(E4M3), wide_s[:blocks(capacity)]
    offsets = torch.tensor(bad, dtype=torch.int32, device="cuda")
    if both:
        fp8.quantize_both(ctx, x, *fp8.empty_rows(M, C), c, sc, offsets=offsets)
    else:
        fp8.quantize_cols(ctx, x, c, sc, offsets=offsets)
    torch.cuda.synchronize()
    ends = np.maximum.accumulate(np.clip(bad, 0, M))
    at = 0
    for a, z in zip(ends[:-1], ends[1:]):
        n, up = z - a, blocks(z - a) * 128
        if n:
            check_quantized(c[at:at + n], sc[at // 128:(at + up) // 128], ref.f64(x)[a:z], 128, 1, "e4m3", False, "a group's columns")
            assert bool((c[at + n:at + up].float() == 0).all())
        at += up
    assert at <= capacity
    assert bool((wide[at:] == 0x55).all()) and bool((wide[:, C:] == 0x55).all()) and bool((wide_s[at // 128:] == -1.0).all())


@pytest.mark.parametrize("offsets", [[0, 30, 30, 170], [200, 330], [5, 5], [300, 300, 300], [0, 0], [129, 128, 131]], ids=str)
@pytest.mark.parametrize("gathered", [False, True], ids=["plain", "gathered"])
def test_quantize_both_makes_every_row(ctx, offsets, gathered):
    """Rows of no group -- ahead of the first one's, from the last offset on -- have their row copy as quantize_rows makes it."""
    M, C = 300, 200
    g = rng("every row", offsets)
    x = torch.randn(M, C, generator=g, device="cuda")
    rows = torch.randint(-1, M + 1, (M,), generator=g, device="cuda", dtype=torch.int32) if gathered else None
    off = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    E = len(offsets) - 1
    q, s = fp8.empty_rows(M, C)
    want_q, want_s = fp8.empty_rows(M, C)
    c, sc = fp8.empty_cols(M, C, E)
    want_c, want_sc = fp8.empty_cols(M, C, E)
    for t in (q, c, want_c):
        t.view(torch.uint8)[:] = 0x55
    for t in (s, sc, want_sc):
        t.fill_(-1.0)
    fp8.quantize_both(ctx, x, q, s, c, sc, rows=rows, offsets=off)
    fp8.quantize_rows(ctx, x, want_q, want_s, rows=rows)
    fp8.quantize_cols(ctx, x, want_c, want_sc, rows=rows, offsets=off)
    assert torch.equal(q.view(torch.uint8), want_q.view(torch.uint8)) and torch.equal(s, want_s)
    assert torch.equal(c.view(torch.uint8), want_c.view(torch.uint8)) and torch.equal(sc, want_sc)


# ---- more elements than 32 bits count ------------------------------------------------------------------------------

def test_quantize_beyond_32_bits(ctx):
    """The ends of matrices of more than 2^31 elements: by rows, with columns, gathered from, and as a stack of weights."""
    R, C = 530048, 4096
    x = torch.zeros(R, C, dtype=torch.bfloat16, device="cuda")
    x[-256:] = torch.randn(256, C, generator=rng("large"), device="cuda") * 3.0
    q, s = fp8.empty_rows(R, C)
    c, sc = fp8.empty_cols(R, C)
    fp8.quantize_rows(ctx, x, q, s)
    same_as_definition(q[-256:], s[-256:], x[-256:], "e4m3", False, 1, 128, "rows")
    q.view(torch.uint8)[-256:] = 0
    fp8.quantize_both(ctx, x, q, s, c, sc)
    same_as_definition(q[-256:], s[-256:], x[-256:], "e4m3", False, 1, 128, "rows with columns")
    same_as_definition(c[-256:], sc[-2:], x[-256:], "e4m3", False, 128, 1, "columns")
    rows = torch.arange(R - 256, R, dtype=torch.int32, device="cuda")
    few = fp8.empty_rows(256, C)
    fp8.quantize_rows(ctx, x, *few, rows=rows)
    same_as_definition(*few, x[-256:], "e4m3", False, 1, 128, "gathered")
    del q, s, c, sc
    stack = x[:128 * 4096].view(128, 4096, C)
    stack[-1, -200:] = x[-200:]
    t, st = fp8.empty_tiles(*stack.shape)
    fp8.quantize_tiles(ctx, stack, t, st)
    same_as_definition(t[-1], st[-1], stack[-1], "e4m3", False, 128, 128, "tiles")


@pytest.mark.parametrize("config,extra", [((2, 256, 1), 0), ((2, 256, 1), 1), ((1, 128, 1), 0), ((1, 64, 2), 0)], ids=str)
def test_results_beyond_32_bits(ctx, config, extra):
    """The last rows of a result of more than 2^31 elements; its other rows keep out of them."""
    M, N, K = 262500, 8192, 200
    g = rng("large result")
    a, b, sa, sb = bytes8(g, (M, K), E4M3), bytes8(g, (N, K), E4M3), scales(g, M, 2), scales(g, blocks(N), 2)
    out = torch.empty(M, N + extra, dtype=torch.bfloat16, device="cuda")[:, :N]
    with fp8.Plan(ctx, M, N, K) as plan:
        plan.set_config(*config)
        plan.run(a, sa, b, sb, out)
        assert plan.last_device_status()[0] == hgemm.OK
    w = ref.values(b, sb, 128, 128)
    for at in (slice(0, 100), slice(M - 300, M)):
        ref.check_product(out[at], ref.values(a[at], sa[at], 1, 128), w, 2, f"{config} {at}")


def test_experts_beyond_32_bits(ctx):
    """The last of 40 experts, whose weight and whose weight gradient begin behind 2^31 elements."""
    E, N, K, M = 40, 8192, 8192, 130
    g = rng("large experts")
    w = torch.full((E, N, K), 0x7F, dtype=torch.uint8, device="cuda").view(E4M3)       # NaN: only the last one may be read
    sb = scales(g, E, blocks(N), blocks(K))
    a, sa = bytes8(g, (M, K), E4M3), scales(g, M, blocks(K))
    last, slast = bytes8(g, (N, K), E4M3, 0.1), sb[-1]
    w[-1].copy_(last)
    offsets = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    offsets[-1] = M
    picked = slice(N - 150, N)
    want_w = ref.values(last, slast, 128, 128)
    for config in ((2, 256, 1), (1, 128, 1)):
        out = torch.full((M, N), float("nan"), device="cuda")
        with fp8.Plan(ctx, M, N, K, groups=E, out_dtype=torch.float32) as plan:
            plan.set_config(*config)
            plan.run(a, sa, w, sb, out, offsets=offsets)
            assert plan.last_device_status()[0] == hgemm.OK
        ref.check_product(out[:, picked], ref.values(a, sa, 1, 128), want_w[picked], blocks(K), f"forward {config}")
    del w
    R = fp8.padded_rows(M, E)
    dy, x = bytes8(g, (R, N), E4M3), bytes8(g, (R, K), E4M3)
    for t in (dy, x):
        t.view(torch.uint8)[M:] = 0
    sy, sx = scales(g, blocks(R), N), scales(g, blocks(R), K)
    p, q = ref.values(dy[:M], sy[:2], 128, 1).T, ref.values(x[:M], sx[:2], 128, 1).T
    for config in ((2, 256, 1), (1, 128, 1)):
        dw = torch.full((E, N, K), float("nan"), dtype=torch.bfloat16, device="cuda")
        with fp8.Plan(ctx, M, N, K, form="weight_grad", groups=E) as plan:
            plan.set_config(*config)
            plan.run(dy, sy, x, sx, dw, offsets=offsets)
            assert plan.last_device_status()[0] == hgemm.OK
        ref.check_product(dw[-1, picked], p[picked], q, 2, f"weight gradient {config}")
        assert not bool(dw[:-1].any())                          # (NaN counts as true)


# ---- the layer as a whole ---------------------------------------------------------------------------------------

def test_gradients_against_differences(ctx):
    """loss = sum(Y * G) for Y = X W^T: the gradients through the 8-bit products against differences of the 64-bit loss.  Operands
    are exact in 8 bits (integers, scale 2^-k), so the products' own errors are those of 32-bit sums."""
    M, N, K = 12, 20, 24
    g = rng("differences")
    X, W, G = (torch.randint(-8, 9, s, generator=g, device="cuda").float() for s in ((M, K), (N, K), (M, N)))

    def rows(t):
        q, s = fp8.empty_rows(*t.shape)
        fp8.quantize_rows(ctx, t, q, s, pow2=True)
        return q, s

    def cols(t):
        q, s = fp8.empty_cols(*t.shape)
        fp8.quantize_cols(ctx, t, q, s, pow2=True)
        return q, s

    wq = fp8.empty_tiles(N, K)
    fp8.quantize_tiles(ctx, W, *wq, pow2=True)
    dX, dW = torch.empty(M, K, device="cuda"), torch.empty(N, K, device="cuda")
    fp8.Plan(ctx, M, N, K, form="input_grad", out_dtype=torch.float32).run(*rows(G), *wq, dX)
    fp8.Plan(ctx, M, N, K, form="weight_grad", out_dtype=torch.float32).run(*cols(G), *cols(X), dW)
    x, w, gg = ref.f64(X), ref.f64(W), ref.f64(G)
    loss = lambda x, w: float(((x @ w.T) * gg).sum())  # noqa: E731
    h = 0.5                                                  # the loss is linear in each operand: differences are exact for any step
    for t, d, at in ((0, dX, [(0, 0), (M - 1, K - 1), (5, 7)]), (1, dW, [(0, 0), (N - 1, K - 1), (11, 3)])):
        for i, j in at:
            up, down = [x.copy(), w.copy()], [x.copy(), w.copy()]
            up[t][i, j] += h
            down[t][i, j] -= h
            assert float(d[i, j]) == pytest.approx((loss(*up) - loss(*down)) / (2 * h), rel=1e-6)


# ---- refusals --------------------------------------------------------------------------------------------------------

def test_refusals(ctx):
    """Wrong arguments raise, and nothing is launched: the result keeps its values."""
    M, N, K = 20, 64, 256
    g = rng("refusals")
    a, w = bytes8(g, (M, K), E4M3), bytes8(g, (N, K), E4M3)
    sa, sb = scales(g, M, 2), scales(g, 1, 2)
    out = torch.full((M, N), 7.0, device="cuda")
    offsets = torch.tensor([0, M], dtype=torch.int32, device="cuda")
    plan = fp8.Plan(ctx, M, N, K, out_dtype=torch.float32)
    bf = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    for args, kw in [
        ((a[:, :255], sa, w, sb, out), {}), ((a.float(), sa, w, sb, out), {}), ((a, sa[:, :1], w, sb, out), {}), ((a, sa.double(), w, sb, out), {}),
        ((a, sa, w[:10], sb, out), {}), ((a, sa, w, sb, bf), {}), ((a, sa, w, sb, out.t().contiguous().t()), {}), ((a.cpu(), sa, w, sb, out), {}),
        ((a, sa, w, sb, out), {"offsets": offsets}), ((a.view(torch.uint8), sa, w, sb, out), {}),
    ]:
        with pytest.raises(ValueError):
            plan.run(*args, **kw)
    grouped = fp8.Plan(ctx, M, N, K, groups=1, out_dtype=torch.float32)
    with pytest.raises(ValueError):
        grouped.run(a, sa, w.unsqueeze(0), sb.unsqueeze(0), out)
    with pytest.raises(ValueError):
        grouped.run(a, sa, w.unsqueeze(0), sb.unsqueeze(0), out, offsets=offsets.long())
    for bad in (dict(form="sideways"), dict(a_dtype=torch.uint8), dict(out_dtype=torch.float64)):
        with pytest.raises(ValueError):
            fp8.Plan(ctx, M, N, K, **bad)
    for shape in ((-1, N, K), (M, 0, K), (M, N, 1 << 23)):
        with pytest.raises(hgemm.HgemmError):
            fp8.Plan(ctx, *shape)
    with pytest.raises(hgemm.HgemmError):
        fp8.Plan(ctx, M, N, K, groups=1025)
    for config in ((2, 128, 1), (2, 256, 2), (1, 256, 1), (1, 8, 1), (1, 64, 3), (3, 64, 1), (1, 64, 16)):
        with pytest.raises(hgemm.HgemmError):
            plan.set_config(*config)
    with pytest.raises(hgemm.HgemmError):
        fp8.Plan(ctx, M, N, K, form="weight_grad").set_config(1, 64, 1)
    # rows that are not 16 bytes apart, a base that is not aligned, C += into a 16-bit result: refused by the library itself
    tight = torch.zeros(M, 250, dtype=torch.uint8, device="cuda").view(E4M3)
    with pytest.raises(hgemm.HgemmError):
        fp8.Plan(ctx, M, N, 250, out_dtype=torch.float32).run(tight, sa, bytes8(g, (N, 250), E4M3), sb, out)
    shifted = torch.zeros(M * 272 + 16, dtype=torch.uint8, device="cuda")[8:8 + M * 272].view(E4M3).view(M, 272)[:, :K]
    with pytest.raises(hgemm.HgemmError):
        plan.run(shifted, sa, w, sb, out)
    with pytest.raises(hgemm.HgemmError):
        fp8.Plan(ctx, M, N, K).run(a, sa, w, sb, bf, accumulate=True)
    x = torch.randn(M, K, device="cuda")
    q, s = fp8.empty_rows(M, K)
    for call in (lambda: fp8.quantize_rows(ctx, x.int(), q, s), lambda: fp8.quantize_rows(ctx, x, q[:3], s), lambda: fp8.quantize_rows(ctx, x, q, s[:, :1]),
                 lambda: fp8.quantize_rows(ctx, x, x, s), lambda: fp8.quantize_rows(ctx, x, q, s, rows=offsets.long()), lambda: fp8.quantize_cols(ctx, x, q, s),
                 lambda: fp8.quantize_cols(ctx, x, q, torch.empty(1, K, device="cuda"), offsets=offsets[:1]), lambda: fp8.quantize_tiles(ctx, x[0], q, s)):
        with pytest.raises(ValueError):
            call()
    torch.cuda.synchronize()
    assert bool((out == 7.0).all())


def test_closed_plans_and_contexts_are_refused():
    """A plan that is closed, or whose context is, raises in every call."""
    with hgemm.Context(0) as c:
        plans = [fp8.Plan(c, 16, 64, 128), fp8.Plan(c, 16, 64, 128)]
        plans[0].close()
    a, sa = fp8.empty_rows(16, 128)
    w, sw = fp8.empty_tiles(64, 128)
    y = torch.full((16, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    for plan in plans:
        for call in (lambda: plan.run(a, sa, w, sw, y), lambda: plan.config, lambda: plan.set_config(1, 16, 1), plan.debug_timeout_probe):
            with pytest.raises(hgemm.HgemmError):
                call()
        assert plan.last_device_status()[0] == hgemm.ERR_INVALID_ARG
        plan.close()
    with pytest.raises(hgemm.HgemmError):
        fp8.quantize_rows(c, torch.zeros(16, 128, device="cuda"), a, sa)
    assert bool((y == 7.0).all())


# ---- the operators together ---------------------------------------------------------------------------------------------

def test_layer_of_experts(ctx):
    """A training step of a layer of experts against the same layer in 64 bits without quantisation, the choice taken as it was made.
    An 8-bit value is within 2^-4 of its element, so a quantised operand is within 2^-4 of the operand's norm at most (about 2^-4 /
    sqrt(3) for spread-out mantissas); at most four such operands, and bf16 results, stand between input and output."""
    from paper_2512_02551_b200.run_experts import ExpertLayer
    T, H, I, E, k = 300, 256, 192, 6, 2
    layer = ExpertLayer(ctx, T, H, I, E, k, seed=5)
    g = rng("layer")
    x, dy = torch.randn(T, H, generator=g, device="cuda").half(), torch.randn(T, H, generator=g, device="cuda")
    y = layer.forward(x)
    dx, dw1, dw2, dlogits = layer.backward(dy)
    assert ctx.last_device_status()[0] == hgemm.OK
    xd, wr, w1, w2 = x.double().requires_grad_(), layer.wr.double().requires_grad_(), layer.w1.double().requires_grad_(), layer.w2.double().requires_grad_()
    p = torch.softmax(xd @ wr.t(), -1).gather(1, layer.indices.long())
    p = p / p.sum(-1, keepdim=True)
    want = torch.zeros(T, H, dtype=torch.float64, device="cuda")
    for e in range(E):
        t, j = torch.nonzero(layer.indices == e, as_tuple=True)
        want = want.index_add(0, t, p[t, j].unsqueeze(-1) * (torch.nn.functional.silu(xd[t] @ w1[e].t()) @ w2[e].t()))
    want.backward(dy.double())
    near = lambda a, b: float((a.double() - b).norm() / b.norm())  # noqa: E731
    bound = 4 * 2.0 ** -4 / 3 ** 0.5
    assert near(y, want) < bound and near(dx, xd.grad) < bound and near(dw1, w1.grad) < bound and near(dw2, w2.grad) < bound

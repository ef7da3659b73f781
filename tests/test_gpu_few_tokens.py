"""The layer of experts for a few tokens on the GPU, against the formula in 64 bits.

Results sit inside guard bands, x's and the weights' rows inside NaN; the tolerance follows from the arithmetic (see ``check``)."""
import ctypes
import os
import subprocess
import sys
import threading
import zlib

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import fp4_reference as ref  # noqa: E402
from paper_2512_02551_b200 import few_tokens, fp4, hgemm, routing  # noqa: E402

DTYPE = {"bf16": torch.bfloat16, "f16": torch.float16}
#: Bits of h against each kind of weights (None: digits).
BITS = {"bf16": 16, "f16": 16, "nvfp4": None, "mxfp4": None}
KINDS = [("bf16", "bf16"), ("f16", "f16"), ("nvfp4", "bf16"), ("nvfp4", "f16"), ("mxfp4", "bf16"), ("mxfp4", "f16")]


@pytest.fixture(scope="module")
def ctx():
    assert torch.cuda.is_available(), "these tests need a B200"
    with hgemm.Context(0) as c:
        yield c


def rng(*key):
    return np.random.default_rng(zlib.crc32(repr(key).encode()))


def wide(t, extra, offset=0):
    """A copy of a matrix or a stack whose rows are `extra` elements further apart than they need be, NaN between them, `offset` elements into its buffer."""
    shape = (*t.shape[:-1], t.shape[-1] + extra)
    buf = torch.full((offset + int(np.prod(shape)) + 8,), float("nan"), dtype=t.dtype, device="cuda")
    v = buf[offset:offset + int(np.prod(shape))].view(shape)[..., :t.shape[-1]]
    v.copy_(t)
    return v


def weights_of(r, shape, kind, extra=0, offset=0):
    """(what the call takes, values in 64 bits)."""
    E, N, K = shape
    if kind in DTYPE:
        w = torch.from_numpy(r.standard_normal(shape) * K ** -0.5).to(DTYPE[kind])
        return wide(w, extra, offset), ref.f64(w)
    code = r.integers(0, 16, shape).astype(np.uint8)
    lo, hi = ((0x28, 0x48) if kind == "nvfp4" else (122, 130))
    s = r.integers(lo, hi, (E, N, ref.blocks(K, kind))).astype(np.uint8)
    factor = (np.exp2(r.integers(-2, 3, E)) * 1.25 / 8 * K ** -0.5).astype(np.float32) if kind == "nvfp4" else np.ones(E, np.float32)
    if kind == "mxfp4":
        s -= np.uint8(np.log2(K) // 2 + 2)
    packed = ref.pack(code)
    pitch = -(-packed.shape[-1] // 16) * 16 + 16 * (extra > 0)
    buf = np.full((E, N, pitch), 0x77, np.uint8)
    buf[..., :packed.shape[-1]] = packed
    q = torch.from_numpy(buf).cuda()[..., :packed.shape[-1]]
    tiles = torch.from_numpy(ref.tiles_from(s, kind)).cuda()
    values = ref.decode(code) * ref.spread(ref.scale_values(s, kind), kind, K) * factor.astype(np.float64)[:, None, None]
    return (q, tiles, torch.from_numpy(factor).cuda()) if kind == "nvfp4" else (q, tiles), values


def silu(u):
    with np.errstate(over="ignore"):
        return u / (1 + np.exp(-u))


def formula(x, w1, w2, indices, weights, gated, bits=16):
    """(y, bound of the error before y's rounding) in 64 bits.

    `bits`: what h is rounded to (2^-bits: a half step, and the factors' products; an fp16 weight against h loses the product of two second parts, as much
    again); None: x and h are sums of digits, off by at most 2^-19 of their largest magnitude.  The contraction over `hidden` adds H numbers in 32
    bits (2^-23 of their magnitudes each covers truncation; with digits, eight times as many, and 8 more); silu changes by at most 1.1 times its argument's error, and its exponential is off by 2^-21 (2 + |u|) of itself; then I, and k, numbers are added."""
    digits = bits is None
    many, lost = (8, 2.0 ** -19) if digits else (1, 0.0)
    T, H = x.shape
    E, I = w1.shape[0], w2.shape[-1]
    y, err = np.zeros((T, H)), np.zeros((T, H))
    for t in range(T):
        for j in range(indices.shape[1]):
            e = indices[t, j]
            if not 0 <= e < E:
                continue
            u = w1[e] @ x[t]
            du = (many * H + 8) * 2.0 ** -23 * (np.abs(w1[e]) @ np.abs(x[t])) + lost * np.abs(x[t]).max() * np.abs(w1[e]).sum(1)
            g = silu(u[:I])
            dg = 1.1 * du[:I] + np.abs(g) * (2 + np.abs(u[:I])) * 2.0 ** -21
            h, dh = (g * u[I:], np.abs(u[I:]) * dg + (np.abs(g) + dg) * du[I:]) if gated else (g, dg)
            dh = dh + (lost * np.abs(h).max() if digits else np.abs(h) * 2.0 ** (1 - bits)) + 2.0 ** -130
            z = w2[e] @ h
            mag = np.abs(w2[e]) @ np.abs(h)
            w = weights[t, j]
            y[t] += w * z
            err[t] += np.abs(w) * (np.abs(w2[e]) @ dh + (many * I + indices.shape[1] + 8) * 2.0 ** -23 * mag)
    return y, err


def check(got, y, err, what=""):
    bound = err + ref.UNIT[got.dtype] * (np.abs(y) + err) + ref.SMALLEST[got.dtype]
    off = np.abs(ref.f64(got) - y)
    bad = ~(off <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.size} off, first at {np.argwhere(bad)[0]}: off {off[bad][0]:.3g}, bound {bound[bad][0]:.3g}"


def case(ctx, kind, dtype, T, H, I, E, k, gated, extra=0, offset=0, indices=None):
    r = rng(kind, dtype, T, H, I, E, k, gated)
    dt = DTYPE[dtype]
    x = torch.from_numpy(r.standard_normal((T, H))).to(dt)
    w1, v1 = weights_of(r, (E, I * (2 if gated else 1), H), kind, extra, offset)
    w2, v2 = weights_of(r, (E, H, I), kind, extra, offset)
    if indices is None:
        indices = np.stack([r.permutation(E)[:k] for _ in range(T)]) if k <= E else r.integers(0, E, (T, k))
    weights = r.random((T, k)).astype(np.float32)
    layer = few_tokens.Layer(ctx, H, I, E, k, weights=kind, activation="swiglu" if gated else "silu", dtype=dt)
    buf = torch.full((offset + T * (H + extra) + 64,), float("nan"), dtype=dt, device="cuda")
    y = buf[offset:offset + T * (H + extra)].view(T, H + extra)[:, :H]
    scratch = layer.empty_scratch(T)
    scratch.fill_(0xFF)                                            # NaN
    xs = wide(x, extra, offset)
    layer.run(xs, w1, w2, torch.tensor(indices, dtype=torch.int32, device="cuda"), torch.from_numpy(weights).cuda(), y, scratch)
    torch.cuda.synchronize()
    keep = torch.ones_like(buf, dtype=torch.bool)
    keep.as_strided(y.shape, y.stride(), y.storage_offset()).fill_(False)
    assert bool(torch.isnan(buf[keep]).all()), "something outside the result was written"
    check(y, *formula(ref.f64(x), v1, v2, indices, weights.astype(np.float64), gated, BITS[kind]), f"{kind} {dtype} {T}x{H}x{I}, {k} of {E}")
    return y


@pytest.mark.parametrize("kind,dtype", KINDS)
@pytest.mark.parametrize("T,k,E", [(1, 1, 1), (1, 8, 16), (2, 2, 5), (8, 2, 3), (9, 1, 1), (17, 2, 2), (33, 4, 7), (64, 2, 3)])
def test_tokens_and_experts(ctx, kind, dtype, T, k, E):
    case(ctx, kind, dtype, T, 256, 192, E, k, True)


@pytest.mark.parametrize("kind,dtype", KINDS)
@pytest.mark.parametrize("H,I", [(1, 1), (7, 9), (16, 8), (64, 100), (129, 77), (256, 33), (333, 520), (1000, 40), (2048, 24), (40, 2050)])
@pytest.mark.parametrize("gated", [False, True])
def test_extents(ctx, kind, dtype, H, I, gated):
    case(ctx, kind, dtype, 3, H, I, 4, 2, gated)


@pytest.mark.parametrize("kind,dtype", KINDS)
@pytest.mark.parametrize("extra,offset", [(1, 0), (2, 0), (8, 0), (0, 1), (0, 2), (3, 5)])
def test_strides_and_alignment(ctx, kind, dtype, extra, offset):
    for H, I in ((96, 130), (131, 65)):
        case(ctx, kind, dtype, 5, H, I, 3, 2, True, extra, offset)


@pytest.mark.parametrize("kind,dtype", KINDS[::2])
def test_choices_outside_twice_and_none(ctx, kind, dtype):
    """Numbers outside the experts count as zero; an expert chosen twice counts twice; a token, or all of them, may have no expert."""
    E = 3
    indices = np.array([[0, 0, 2], [-1, 5, 1], [E, -7, 1 << 30], [2, 2, 2], [1, 0, -(1 << 31)]], dtype=np.int64)
    case(ctx, kind, dtype, 5, 128, 64, E, 3, True, indices=indices)
    y = case(ctx, kind, dtype, 2, 128, 64, E, 3, False, indices=np.full((2, 3), -1))
    assert bool((y == 0).all())


@pytest.mark.parametrize("kind,dtype", [("nvfp4", "bf16"), ("bf16", "bf16")])
def test_most_choices(ctx, kind, dtype):
    case(ctx, kind, dtype, 64, 64, 48, 40, 32, True)
    case(ctx, kind, dtype, 64, 48, 40, 1, 32, False, indices=np.zeros((64, 32), np.int64))


@pytest.mark.parametrize("kind,dtype", KINDS)
@pytest.mark.parametrize("T,k,E,H,I", [(1, 3, 5, 40, 300), (2, 1, 4, 24, 500), (61, 7, 50, 24, 200), (64, 5, 9, 600, 33), (20, 6, 40, 1200, 65)])
def test_few_outputs_for_many_choices(ctx, kind, dtype, T, k, E, H, I):
    """Outputs that several CTAs share, by one choice each and by more than their warps take at once; numbers of choices that are not multiples of
    anything, some of them of no expert."""
    r = rng("few outputs", T, k, E)
    indices = np.where(r.random((T, k)) < 0.1, -1, r.integers(0, E, (T, k)))
    case(ctx, kind, dtype, T, H, I, E, k, False, indices=indices)


def test_many_experts_and_rounds(ctx):
    """More tiles than warps: every warp walks on to further experts."""
    case(ctx, "nvfp4", "bf16", 24, 512, 1024, 96, 8, True)
    case(ctx, "f16", "f16", 24, 512, 1024, 64, 4, False)


@pytest.mark.parametrize("kind,dtype", KINDS)
@pytest.mark.parametrize("H", [4097, 4128, 4224, 5120, 8193])
def test_long_hidden(ctx, kind, dtype, H):
    """x in more pieces than one (16-bit weights: 4096 elements at a time, the last piece of less than a run of chunks among them), and longer than a pass of the threads that make digits."""
    case(ctx, kind, dtype, 3, H, 72, 3, 2, H % 2 == 0)
    case(ctx, kind, dtype, 10, H, 40, 2, 1, H % 2 == 1, *((1, 0), (2, 0), (8, 8))[H % 3])


@pytest.mark.parametrize("kind,dtype,gated", [("bf16", "bf16", True), ("f16", "f16", False)])
def test_long_hidden_in_several_rounds(ctx, kind, dtype, gated):
    """More groups of rows than CTAs, in pieces: from round to round of one expert's tokens, on to the next's, and the rest shared."""
    case(ctx, kind, dtype, 64, 4232, 640 if gated else 1280, 4, 4, gated, indices=rng("rounds", kind).integers(0, 4, (64, 4)))


@pytest.mark.parametrize("kind,dtype", KINDS[::2])
def test_as_many_experts_as_there_may_be(ctx, kind, dtype):
    r = rng("experts", kind)
    case(ctx, kind, dtype, 64, 48, 24, 1024, 32, True, indices=r.integers(0, 1024, (64, 32)))
    case(ctx, kind, dtype, 2, 48, 24, 1024, 3, False, indices=np.array([[1023, 0, 1023], [-1, 1022, 1024]]))


@pytest.mark.parametrize("kind", ["bf16", "nvfp4", "mxfp4"])
def test_stacks_beyond_32_bits(ctx, kind):
    """Stacks of more than 2^31 elements (16-bit) or bytes (4-bit); the last experts, the first and one between are chosen."""
    E, H, I, k, gated = (600, 2048, 1800, 3, False) if kind == "bf16" else (1024, 2048, 1100, 3, True)
    chosen = np.array([[E - 1, 0, E // 2], [E - 2, E - 1, 1]])
    g = torch.Generator(device="cuda").manual_seed(3)
    held, values = [], []
    for shape in ((E, 2 * I if gated else I, H), (E, H, I)):
        K = shape[-1]
        if kind == "bf16":
            w = torch.zeros(shape, dtype=torch.bfloat16, device="cuda")
            for e in np.unique(chosen):
                w[e] = (torch.randn(shape[1:], generator=g, device="cuda") * K ** -0.5).bfloat16()
            held.append(w)
            values.append({e: ref.f64(w[e]) for e in np.unique(chosen)})
        else:
            n = -(-K // 2)
            q = torch.randint(0, 256, (*shape[:-1], -(-n // 16) * 16), dtype=torch.uint8, generator=g, device="cuda")[..., :n]
            tiles = torch.randint(*((0x28, 0x40) if kind == "nvfp4" else (118, 124)), fp4._scales_shape(shape, kind), dtype=torch.uint8, generator=g, device="cuda")
            held.append((q, tiles, torch.full((E,), 0.0625, device="cuda")) if kind == "nvfp4" else (q, tiles))
            values.append({e: ref.values(q[e], tiles[e], K, kind, 0.0625 if kind == "nvfp4" else 1.0) for e in np.unique(chosen)})
        assert max(t.numel() for t in ([held[-1]] if kind == "bf16" else held[-1][:1])) > (1 << 31 if len(held) == 1 else 1 << 30)
    x = torch.randn(2, H, generator=g, device="cuda").bfloat16()
    weights = torch.rand(2, k, generator=g, device="cuda")
    layer = few_tokens.Layer(ctx, H, I, E, k, weights=kind, activation="swiglu" if gated else "silu")
    y = torch.empty_like(x)
    layer.run(x, *held, torch.tensor(chosen, dtype=torch.int32, device="cuda"), weights, y, layer.empty_scratch(2))
    order = np.unique(chosen)                                      # the formula on the chosen ones alone
    check(y, *formula(ref.f64(x), np.stack([values[0][e] for e in order]), np.stack([values[1][e] for e in order]), np.searchsorted(order, chosen), ref.f64(weights), gated, BITS[kind]), kind)


@pytest.mark.parametrize("kind,dtype", KINDS[::2])
@pytest.mark.parametrize("H,I", [(5120, 1536), (7168, 512)])
def test_widths_of_large_layers(ctx, kind, dtype, H, I):
    case(ctx, kind, dtype, 4, H, I, 3, 2, True)


FIRST_CALL = """
import sys
sys.path[:0] = %r
import test_gpu_few_tokens as few
from paper_2512_02551_b200 import hgemm
with hgemm.Context(0) as ctx:
    few.case(ctx, *%r)
"""


@pytest.mark.parametrize("kind,T,k,E,H", [("bf16", 1, 2, 4, 2688), ("f16", 1, 2, 4, 2700), ("bf16", 2, 3, 5, 2816), ("bf16", 1, 1, 1, 2880), ("f16", 1, 2, 4, 2944), ("bf16", 16, 8, 128, 2624)])
def test_a_process_first_call(kind, T, k, E, H):
    """Sizes around the shared memory that a kernel has without asking, each as the first call of a process: nothing has raised the limit before."""
    args = (kind, kind, T, H, 24, E, k, False)
    here = os.path.dirname(os.path.abspath(__file__))
    done = subprocess.run([sys.executable, "-c", FIRST_CALL % ([here, os.path.dirname(here)], args)], capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, done.stderr[-2000:]


def test_threads_with_contexts_of_their_own():
    """Calls of different sizes from two threads, each with its own context, stream and scratch memory: none changes what the other's launch may have."""
    H, I, E, k, N = 64, 32, 16, 8, 20000
    m1, m2 = (torch.randn(*s, device="cuda").bfloat16() for s in ((E, I, H), (E, H, I)))
    torch.cuda.synchronize()
    refused, gate = [], threading.Barrier(2)

    def decode(T):
        stream = torch.cuda.Stream()
        with hgemm.Context(0) as own, torch.cuda.stream(stream):
            layer = few_tokens.Layer(own, H, I, E, k, weights="bf16", activation="silu")
            x, scratch = torch.ones(T, H, device="cuda").bfloat16(), layer.empty_scratch(T)
            idx, w, y = (torch.arange(T * k, device="cuda") % E).int().view(T, k), torch.ones(T, k, device="cuda"), torch.empty_like(x)
            p = ctypes.c_void_p
            ws = [few_tokens.Weights(m.data_ptr(), m.stride(1), None, None) for m in (m1, m2)]
            args = [own._h, ctypes.byref(layer._desc), ctypes.c_int64(T), p(x.data_ptr()), ctypes.c_int64(H), ctypes.byref(ws[0]), ctypes.byref(ws[1]), p(idx.data_ptr()), p(w.data_ptr()),
                    p(y.data_ptr()), ctypes.c_int64(H), p(scratch.data_ptr()), ctypes.c_int64(scratch.numel()), p(stream.cuda_stream)]
            call = few_tokens.lib().hgemm_few_tokens               # the calls themselves, so that they meet
            gate.wait()
            refused.append(sum(call(*args) != hgemm.OK for _ in range(N)))
            stream.synchronize()

    threads = [threading.Thread(target=decode, args=(T,)) for T in (16, 32)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert refused == [0, 0], f"refused calls of {N} each: {refused}"


#: What is lost of x and h, as a part of their largest magnitude (digits: the remainder, see the header) or, for h of 16-bit weights, of itself (two roundings to bf16).
LOST = {"nvfp4": 2.0 ** -19, "mxfp4": 2.0 ** -22, "bf16": 2.0 ** -16, "f16": 2.0 ** -16}


def simple_weights(w, kind):
    """What the call takes of a stack of -1, 0 and 1."""
    if kind in DTYPE:
        return torch.from_numpy(w).to(DTYPE[kind]).cuda()
    packed = ref.pack(np.where(w < 0, 10, np.where(w > 0, 2, 0)).astype(np.uint8))
    n = packed.shape[-1]
    q = torch.from_numpy(np.pad(packed, ((0, 0), (0, 0), (0, -n % 16 + 16)))).cuda()[..., :n]
    one = np.full((*w.shape[:-1], ref.blocks(w.shape[-1], kind)), 0x38 if kind == "nvfp4" else 127, np.uint8)
    return (q, torch.from_numpy(ref.tiles_from(one, kind)).cuda(), *([torch.ones(w.shape[0], device="cuda")] if kind == "nvfp4" else []))


@pytest.mark.parametrize("kind,dtype", KINDS)
def test_neighbouring_values_keep_their_difference(ctx, kind, dtype):
    """Results that are the small differences of nearly equal values of h, so that the last digits of h are all there is.  u = 1.5 + m 2^-16 with m < 16 is exact (one large and one
    small element of x, weights of 1), and the gate the same throughout, so that h differs by silu(1.5) times u's differences but for a rounding of each (2^-24) and what is lost of
    it; a common error of silu (2^-21 (2 + 1.5), see ``formula``) is one of the difference.  The sums are exact: two digits each, multiples of the last digit's step."""
    r = rng("neighbours", kind, dtype)
    H, I, T = 64, 96, 3
    x = np.zeros((T, H))
    x[:, 0] = 1.5
    x[:, 32:] = r.integers(1, 16, (T, H - 32)) * 2.0 ** -16
    w1, w2 = np.zeros((1, 2 * I, H)), np.zeros((1, H, I))
    w1[0, :, 0] = 1
    w1[0, np.arange(I, 2 * I), r.integers(32, H, I)] = 1
    for n in range(H):
        a, b = r.permutation(I)[:2]
        w2[0, n, a], w2[0, n, b] = 1, -1
    xs = torch.from_numpy(x).to(DTYPE[dtype])
    assert np.array_equal(ref.f64(xs), x)
    layer = few_tokens.Layer(ctx, H, I, 1, 1, weights=kind, dtype=DTYPE[dtype])
    y = torch.empty(T, H, dtype=DTYPE[dtype], device="cuda")
    layer.run(xs.cuda(), simple_weights(w1, kind), simple_weights(w2, kind), torch.zeros(T, 1, dtype=torch.int32, device="cuda"), torch.ones(T, 1, device="cuda"), y, layer.empty_scratch(T))
    h = silu(1.5) * (x @ w1[0, I:].T)
    want = h @ w2[0].T
    check(y, want, 2 * (LOST[kind] + 2.0 ** -24) * np.abs(h).max() + 3.5 * 2.0 ** -21 * np.abs(want), f"{kind} {dtype}")


@pytest.mark.parametrize("kind,dtype", KINDS)
@pytest.mark.parametrize("large", [2.0 ** 4, 2.0 ** 8, 2.0 ** 11])
def test_small_values_beside_a_large_channel(ctx, kind, dtype, large):
    """One element of x far larger than the others, which half of the rows of W1 do not look at: what the others keep."""
    r = rng("large channel", kind, dtype, large)
    T, H, I = 3, 192, 80
    x = r.standard_normal((T, H))
    x[:, 5] = large * (1 + r.random(T))
    x = torch.from_numpy(x).to(DTYPE[dtype])
    w1 = np.where(r.random((1, 2 * I, H)) < 0.3, r.choice([-1.0, 1.0], (1, 2 * I, H)), 0.0)
    w1[0, :, 5] = r.random(2 * I) < 0.02
    w2 = r.choice([-1.0, 0.0, 1.0], (1, H, I))
    layer = few_tokens.Layer(ctx, H, I, 1, 1, weights=kind, dtype=DTYPE[dtype])
    y = torch.empty(T, H, dtype=DTYPE[dtype], device="cuda")
    weight = np.full((T, 1), 2.0 ** -8)
    layer.run(x.cuda(), simple_weights(w1, kind), simple_weights(w2, kind), torch.zeros(T, 1, dtype=torch.int32, device="cuda"), torch.full((T, 1), 2.0 ** -8, device="cuda"), y,
              layer.empty_scratch(T))
    check(y, *formula(ref.f64(x), w1, w2, np.zeros((T, 1), int), weight, True, BITS[kind]), f"{kind} {dtype} {large}")


@pytest.mark.parametrize("kind", ["nvfp4", "mxfp4"])
@pytest.mark.parametrize("e", [100, 112, 118, 122])
def test_digits_of_the_smallest_numbers(ctx, kind, e):
    """Magnitudes near fp32's smallest: what is lost of x is at most 2^-127 where that is more than its part of the largest; the weights bring the results back."""
    r = rng("smallest", kind, e)
    T, H, I = 4, 80, 48
    x = torch.from_numpy(r.standard_normal((T, H)) * 2.0 ** -e).bfloat16()
    w1, w2 = r.choice([-1.0, 0.0, 1.0], (1, I, H)), r.choice([-1.0, 0.0, 1.0], (1, H, I))
    m1 = list(simple_weights(w1, kind))
    if kind == "nvfp4":
        m1[2] = m1[2] * 2.0 ** 60
    else:
        m1[1] = torch.where(m1[1] == 127, 187, m1[1])               # scales of 2^60
    layer = few_tokens.Layer(ctx, H, I, 1, 1, weights=kind, activation="silu")
    y = torch.empty(T, H, dtype=torch.bfloat16, device="cuda")
    layer.run(x.cuda(), tuple(m1), simple_weights(w2, kind), torch.zeros(T, 1, dtype=torch.int32, device="cuda"), torch.ones(T, 1, device="cuda"), y, layer.empty_scratch(T))
    want, err = formula(ref.f64(x), w1 * 2.0 ** 60, w2, np.zeros((T, 1), int), np.ones((T, 1)), False, None)
    err = err + 1.1 * 2.0 ** (60 - 127) * (np.abs(w2[0]) @ np.abs(w1[0]).sum(1)) * (e > 100)
    check(y, want, err, f"{kind} 2^-{e}")


def test_infinite_and_nan_inputs_stay_in_their_token(ctx):
    for kind, dtype in KINDS:
        r = rng(kind, dtype)
        dt = DTYPE[dtype]
        w1, _ = weights_of(r, (4, 64, 128), kind)
        w2, _ = weights_of(r, (4, 128, 32), kind)
        x = torch.randn(6, 128, device="cuda").to(dt)
        layer = few_tokens.Layer(ctx, 128, 32, 4, 2, weights=kind, dtype=dt)
        idx, w = torch.tensor([[0, 1]] * 6, dtype=torch.int32, device="cuda"), torch.full((6, 2), 0.5, device="cuda")
        clean, y, s = torch.empty_like(x), torch.empty_like(x), layer.empty_scratch(6)
        layer.run(x, w1, w2, idx, w, clean, s)
        x[1, 5], x[4, 100] = float("nan"), float("inf")
        layer.run(x, w1, w2, idx, w, y, s)
        rest = [0, 2, 3, 5]
        assert torch.equal(y[rest], clean[rest])
        assert not torch.isfinite(y[1].float()).any() and not torch.isfinite(y[4].float()).all()


def test_large_h_and_small_x(ctx):
    """h beyond fp16's range, and x among its smallest numbers: no range is lost on the way."""
    for kind, dtype, scale in (("f16", "f16", 2.0 ** 7), ("nvfp4", "f16", 2.0 ** 7), ("mxfp4", "f16", 2.0 ** -14), ("f16", "f16", 2.0 ** -14), ("bf16", "bf16", 2.0 ** -60), ("nvfp4", "bf16", 2.0 ** -60)):
        r = rng(kind, dtype, 3)
        dt = DTYPE[dtype]
        w1, v1 = weights_of(r, (2, 128, 64), kind)
        w2, v2 = weights_of(r, (2, 64, 64), kind)
        x = torch.from_numpy(r.standard_normal((4, 64)) * scale * 8).to(dt)
        layer = few_tokens.Layer(ctx, 64, 64, 2, 1, weights=kind, dtype=dt)
        idx, w = np.array([[0], [1], [0], [1]]), np.full((4, 1), 2.0 ** -12 if scale > 1 else 1.0, np.float32)
        y = torch.empty(4, 64, dtype=dt, device="cuda")
        layer.run(x.cuda(), w1, w2, torch.tensor(idx, dtype=torch.int32, device="cuda"), torch.from_numpy(w).cuda(), y, layer.empty_scratch(4))
        check(y, *formula(ref.f64(x), v1, v2, idx, w.astype(np.float64), True, BITS[kind]), f"{kind} {dtype} {scale}")


def test_with_the_quantiser_and_the_router(ctx):
    """As a decoding step uses it: routed by the library, weights made by its quantiser."""
    T, H, I, E, k = 11, 320, 136, 12, 3
    g = torch.Generator(device="cuda").manual_seed(2)
    for fmt in ("nvfp4", "mxfp4"):
        ops = []
        for shape in ((E, 2 * I, H), (E, H, I)):
            w = torch.randn(*shape, generator=g, device="cuda") * shape[-1] ** -0.5
            f = None
            if fmt == "nvfp4":
                f = torch.empty(E, device="cuda")
                fp4.tensor_factor(ctx, w, f)
            q, s = fp4.empty_rows(*shape, format=fmt)
            fp4.quantize_rows(ctx, w, q, s, factor=f, format=fmt)
            back = torch.empty_like(w)
            fp4.dequantize(ctx, q, s, back, factor=f, format=fmt)
            ops.append(((q, s) if f is None else (q, s, f), ref.f64(back)))
        router = routing.Router(ctx, E, k, score="softmax", renormalize=True)
        logits = torch.randn(T, E, generator=g, device="cuda")
        weights, indices = torch.empty(T, k, device="cuda"), torch.empty(T, k, dtype=torch.int32, device="cuda")
        x = torch.randn(T, H, generator=g, device="cuda").bfloat16()
        y = torch.empty_like(x)
        layer = few_tokens.Layer(ctx, H, I, E, k, weights=fmt)
        router.forward(logits, weights, indices)
        layer.run(x, ops[0][0], ops[1][0], indices, weights, y, layer.empty_scratch(T))
        check(y, *formula(ref.f64(x), ops[0][1], ops[1][1], indices.cpu().numpy(), ref.f64(weights), True, None), fmt)


def test_captured_replayed_and_at_once(ctx):
    """Two captured layers with scratch memory of their own, replayed on two streams at once and over and over, on new inputs: the bits of single calls."""
    r = rng(8)
    E, H, I, k, T = 8, 512, 256, 2, 7
    w1, _ = weights_of(r, (E, 2 * I, H), "nvfp4")
    w2, _ = weights_of(r, (E, H, I), "nvfp4")
    layer = few_tokens.Layer(ctx, H, I, E, k)
    x = torch.randn(T, H, device="cuda").bfloat16()
    idx, w = torch.zeros(T, k, dtype=torch.int32, device="cuda"), torch.rand(T, k, device="cuda")
    ys, scratches, graphs = [torch.empty_like(x) for _ in range(2)], [layer.empty_scratch(T) for _ in range(2)], []
    run = lambda i: layer.run(x, w1, w2, idx, w, ys[i], scratches[i])  # noqa: E731
    run(0)
    torch.cuda.synchronize()
    for i in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[i]):
            run(i)
            run(i)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for n in range(4):
        x.copy_(torch.randn(T, H, device="cuda"))
        idx.copy_(torch.from_numpy(r.integers(-1, E, (T, k))))
        torch.cuda.synchronize()
        for _ in range(20):
            for i in range(2):
                with torch.cuda.stream(streams[i]):
                    graphs[i].replay()
        torch.cuda.synchronize()
        got = [y.clone() for y in ys]
        run(0)
        assert torch.equal(got[0], ys[0]) and torch.equal(got[1], ys[0])


@pytest.mark.parametrize("kind", ["nvfp4", "mxfp4", "bf16"])
def test_steps_in_a_row(ctx, kind):
    """The router's choices, the weights and x are overwritten right ahead of each step and right behind it, by kernels that start before the ones ahead of them end:
    the bits of steps that wait for each other."""
    T, H, I, E, k, N = 16, 512, 256, 16, 4, 12
    g = torch.Generator(device="cuda").manual_seed(5)
    draw = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    w1s, w2s, ls, xs = [draw(E, 2 * I, H) * H ** -0.5 for _ in range(3)], [draw(E, H, I) * I ** -0.5 for _ in range(3)], [draw(T, E) for _ in range(N)], [draw(T, H).bfloat16() for _ in range(N)]
    if kind == "bf16":
        held = [torch.empty(E, 2 * I, H, dtype=torch.bfloat16, device="cuda"), torch.empty(E, H, I, dtype=torch.bfloat16, device="cuda")]
    else:
        held = [(*fp4.empty_rows(*s, format=kind), torch.ones(E, device="cuda") if kind == "nvfp4" else None) for s in ((E, 2 * I, H), (E, H, I))]
    router, layer = routing.Router(ctx, E, k, score="softmax", renormalize=True), few_tokens.Layer(ctx, H, I, E, k, weights=kind)
    weights, indices, x, scratch = torch.empty(T, k, device="cuda"), torch.empty(T, k, dtype=torch.int32, device="cuda"), torch.empty(T, H, dtype=torch.bfloat16, device="cuda"), layer.empty_scratch(T)

    def step(n, y, wait):
        for w, h in ((w1s[n % 3], held[0]), (w2s[n % 3], held[1])):
            if kind == "bf16":
                h.copy_(w)
            else:
                fp4.quantize_rows(ctx, w, h[0], h[1], factor=h[2], format=kind)
        x.copy_(xs[n])
        wait()
        router.forward(ls[n], weights, indices)
        wait()
        layer.run(x, *held, indices, weights, y, scratch)
        wait()

    ys, zs = [torch.empty_like(x) for _ in range(N)], [torch.empty_like(x) for _ in range(N)]
    for n in range(N):
        step(n, ys[n], torch.cuda.synchronize)
    for _ in range(5):
        for n in range(N):
            step(n, zs[n], lambda: None)
        assert all(torch.equal(a, b) for a, b in zip(ys, zs))
    assert ctx.last_device_status()[0] == hgemm.OK


@pytest.mark.parametrize("kind", ["nvfp4", "mxfp4", "bf16", "f16"])
@pytest.mark.parametrize("T,k", [(1, 1), (1, 4), (3, 2)])
def test_steps_of_few_ctas(ctx, kind, T, k):
    """Steps of launches that leave most SMs without a CTA, so that an SM sees the same places of memory again after steps that it had no part in: choices, weights and x change with
    every step, launched one by one and replayed from a graph; the bits of steps that wait for each other."""
    H, I, E, N = 72, 40, 16, 60
    r = rng("few ctas", kind, T, k)
    dt = torch.float16 if kind == "f16" else torch.bfloat16
    w1, _ = weights_of(r, (E, 2 * I, H), kind)
    w2, _ = weights_of(r, (E, H, I), kind)
    layer = few_tokens.Layer(ctx, H, I, E, k, weights=kind, dtype=dt)
    xs, ws = torch.from_numpy(r.standard_normal((N, T, H))).to(dt).cuda(), torch.from_numpy(r.random((N, T, k)).astype(np.float32)).cuda()
    ids = torch.from_numpy(r.integers(-1, E, (N, T, k)).astype(np.int32)).cuda()
    x, w, idx, scratch = torch.empty_like(xs[0]), torch.empty_like(ws[0]), torch.empty_like(ids[0]), layer.empty_scratch(T)
    y = torch.empty_like(x)

    def steps(launch, wait):
        out = torch.empty_like(xs)
        for n in range(N):
            x.copy_(xs[n])
            w.copy_(ws[n])
            idx.copy_(ids[n])
            wait()
            launch()
            wait()
            out[n].copy_(y)
        torch.cuda.synchronize()
        return out

    run = lambda: layer.run(x, w1, w2, idx, w, y, scratch)  # noqa: E731
    want = steps(run, torch.cuda.synchronize)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for launch in (run, graph.replay):
        for _ in range(3):
            assert torch.equal(steps(launch, lambda: None), want)
    assert ctx.last_device_status()[0] == hgemm.OK


def test_no_tokens(ctx):
    layer = few_tokens.Layer(ctx, 64, 64, 2, 1, weights="bf16", dtype=torch.bfloat16, activation="silu")
    w = torch.zeros(2, 64, 64, dtype=torch.bfloat16, device="cuda")
    x = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda")
    layer.run(x, w, w, torch.empty(0, 1, dtype=torch.int32, device="cuda"), torch.empty(0, 1, device="cuda"), x.clone(), layer.empty_scratch(0))


def test_refusals(ctx):
    with pytest.raises(ValueError):
        few_tokens.Layer(ctx, 64, 64, 2, 1, weights="int4")
    with pytest.raises(ValueError):
        few_tokens.Layer(ctx, 64, 64, 2, 1, weights="f16", dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        few_tokens.Layer(ctx, 64, 64, 2, 33)
    layer = few_tokens.Layer(ctx, 64, 64, 2, 1, weights="bf16", activation="silu")
    with pytest.raises(ValueError):
        layer.empty_scratch(65)
    new = lambda *s, dtype=torch.bfloat16: torch.zeros(*s, dtype=dtype, device="cuda")  # noqa: E731
    x, w, idx, wt, s = new(3, 64), new(2, 64, 64), new(3, 1, dtype=torch.int32), new(3, 1, dtype=torch.float32), layer.empty_scratch(3)
    layer.run(x, w, w, idx, wt, x.clone(), s)
    for bad in (dict(x=new(3, 63)), dict(x=x.half()), dict(w1=w.half()), dict(w2=new(2, 64, 65)), dict(indices=idx.long()), dict(weights=wt.half()), dict(y=new(2, 64)), dict(w1=(w, w))):
        with pytest.raises((ValueError, AttributeError)):
            layer.run(**{**dict(x=x, w1=w, w2=w, indices=idx, weights=wt, y=x.clone(), scratch=s), **bad})
    with pytest.raises(hgemm.HgemmError):
        layer.run(x, w, w, idx, wt, x.clone(), layer.empty_scratch(2))                    # too little scratch memory
    with pytest.raises(hgemm.HgemmError):
        layer.run(new(65, 64), w, w, new(65, 1, dtype=torch.int32), new(65, 1, dtype=torch.float32), new(65, 64), layer.empty_scratch(64))
    L, d = few_tokens.lib(), layer._desc
    m = few_tokens.Weights(w.data_ptr(), 64, None, None)
    args = [ctypes.byref(d), 3, x.data_ptr(), 64, ctypes.byref(m), ctypes.byref(m), idx.data_ptr(), wt.data_ptr(), x.data_ptr(), 64, s.data_ptr(), s.numel(), None]
    for i, v in ((0, None), (1, -1), (1, 65), (2, None), (2, x.data_ptr() + 1), (3, 63), (4, None), (4, ctypes.byref(few_tokens.Weights(None, 64, None, None))),
                 (4, ctypes.byref(few_tokens.Weights(w.data_ptr(), 63, None, None))), (4, ctypes.byref(few_tokens.Weights(w.data_ptr() + 1, 64, None, None))),
                 (5, ctypes.byref(few_tokens.Weights(w.data_ptr(), 64, w.data_ptr(), None))), (5, ctypes.byref(few_tokens.Weights(w.data_ptr(), 64, None, wt.data_ptr()))),
                 (6, None), (6, idx.data_ptr() + 2), (7, None), (8, None), (8, x.data_ptr() + 1), (9, 63), (10, None), (10, s.data_ptr() + 8), (11, 16)):
        assert L.hgemm_few_tokens(ctx._h, *[v if j == i else a for j, a in enumerate(args)]) == hgemm.ERR_INVALID_ARG, (i, v)

"""Measured cases of the 4-bit operands with block scales (their quantiser, the products on them) and of a layer of experts for a few tokens.

Four operators.  "quantize" turns activations, gradients or weights into 4-bit values (e2m1: 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives) with one
scale for each block along the contracted dimension, and back into the values that they stand for; "product" is a linear layer's
forward product, its input gradient or its weight gradient on such operands; "experts" is the same with rows sorted by expert and one weight for each
expert; "layer" is both products of a layer of experts, its activation and the weighted sum over each token's choices, for the few tokens of
a decoding step.

Formats: "nvfp4" has blocks of 16 with an e4m3 scale each and one 32-bit factor for the whole tensor, the smallest power of two that keeps every scale in
e4m3's range; "mxfp4" has blocks of 32 with a power of two each.

Inputs: activations are normal with a few large channels, weights normal / sqrt(inputs), gradients normal and small, routing weights positive with a sum of
one.  Sizes are powers of two from 64 to 16384 and odd numbers between them.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BLOCK = {"nvfp4": 16, "mxfp4": 32}
GROUP = 128                 # rows of a scale tile; each expert's rows start at a multiple of it in a column copy
FP8_MAX = 448.0
TINY = 2.0 ** -100          # a tensor factor below this counts as zero


# ---- cases ---------------------------------------------------------------------------------------------------------------

def listed():
    return [
        # quantize: one decoding batch's activations before a projection, checked by their values; latency counts
        {"name": "quantize rows 24x4096", "op": "quantize", "blocks": "rows", "rows": 24, "cols": 4096, "type": "bf16", "format": "nvfp4", "top": 0, "experts": 0},
        # ... a training batch's activations, needed along rows (forward) and along columns (weight gradient); odd row count
        {"name": "quantize both 8191x4096", "op": "quantize", "blocks": "both", "rows": 8191, "cols": 4096, "type": "bf16", "format": "nvfp4", "top": 0, "experts": 0},
        # ... tokens gathered into expert order, both copies, each expert's blocks its own
        {"name": "quantize experts 4096x4x2048 of 32", "op": "quantize", "blocks": "both", "rows": 4096, "cols": 2048, "type": "f16", "format": "mxfp4", "top": 4, "experts": 32},
        # product: a projection while decoding a few sequences: the weights' bytes bound it
        {"name": "forward 7x8192x4096", "op": "product", "form": "forward", "M": 7, "N": 8192, "K": 4096, "out": "bf16", "format": "nvfp4"},
        # ... a prompt of 1000 tokens, result in the library's fp16
        {"name": "forward 1000x4096x4096", "op": "product", "form": "forward", "M": 1000, "N": 4096, "K": 4096, "out": "f16", "format": "mxfp4"},
        # ... the largest square of the benchmark's middle grid: the tensor cores bound it
        {"name": "forward 8192x8192x8192", "op": "product", "form": "forward", "M": 8192, "N": 8192, "K": 8192, "out": "bf16", "format": "nvfp4"},
        # ... training: gradient of the weights, kept in 32 bits, sizes off every tile
        {"name": "weight_grad 8000x4096x2000", "op": "product", "form": "weight_grad", "M": 8000, "N": 4096, "K": 2000, "out": "f32", "format": "nvfp4"},
        # experts: a short prompt, 64 tokens of 8 choices over 64 experts: about eight rows for each weight matrix
        {"name": "experts forward 64x8 of 64", "op": "experts", "form": "forward", "tokens": 64, "top": 8, "experts": 64, "N": 2048, "K": 2048, "out": "bf16", "format": "nvfp4"},
        # ... training: 8192 tokens of 4 choices over 32 experts, gradient of each expert's weights
        {"name": "experts weight_grad 8192x4 of 32", "op": "experts", "form": "weight_grad", "tokens": 8192, "top": 4, "experts": 32, "N": 2048, "K": 2048, "out": "bf16", "format": "mxfp4"},
        # layer: one sequence's next token, eight experts read out of 64
        {"name": "layer 1 token nvfp4", "op": "layer", "tokens": 1, "top": 8, "experts": 64, "hidden": 2048, "inner": 1024, "weights": "nvfp4", "gated": True, "type": "bf16"},
        # ... 16 sequences' next tokens: nearly every expert has a few; 4-bit weights
        {"name": "layer 16 tokens nvfp4", "op": "layer", "tokens": 16, "top": 8, "experts": 64, "hidden": 2048, "inner": 1024, "weights": "nvfp4", "gated": True, "type": "bf16"},
        # ... 5 sequences, weights in 16 bits
        {"name": "layer 5 tokens bf16", "op": "layer", "tokens": 5, "top": 4, "experts": 32, "hidden": 2048, "inner": 1000, "weights": "bf16", "gated": False, "type": "bf16"},
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["quantize", "product", "product", "experts", "experts", "layer", "layer"])
    fmt = rng.choice(list(BLOCK))
    if op == "quantize":
        blocks, experts = rng.choice(["rows", "both"]), rng.choice([0, 0, 8, 32, 60])
        top = rng.choice([1, 2, 4]) if experts else 0
        cols = _log(rng, 64, 8192)
        rows = _log(rng, 1, min(16384, (8191 * 4096) // (cols * max(1, top))))
        return {"op": op, "blocks": blocks, "rows": rows, "cols": cols, "type": rng.choice(list(TYPES)), "format": fmt, "top": top, "experts": experts}
    if op == "product":
        form = rng.choice(["forward", "forward", "input_grad", "weight_grad"])
        return {"op": op, "form": form, "M": _log(rng, 1, 8192), "N": _log(rng, 64, 8192), "K": _log(rng, 64, 8192), "out": rng.choice(list(TYPES)), "format": fmt}
    if op == "experts":
        form = rng.choice(["forward", "input_grad", "weight_grad"])
        return {"op": op, "form": form, "tokens": _log(rng, 1, 8192), "top": rng.choice([1, 2, 4, 8]), "experts": rng.choice([8, 16, 32, 48, 64]), "N": _log(rng, 64, 2048),
                "K": _log(rng, 64, 2048), "out": rng.choice(list(TYPES)), "format": fmt}
    weights = rng.choice(["nvfp4", "mxfp4", "bf16", "f16"])
    return {"op": op, "tokens": _log(rng, 1, 32), "top": rng.choice([1, 2, 4, 8]), "experts": rng.choice([8, 16, 32, 60, 64]), "hidden": _log(rng, 64, 2048), "inner": _log(rng, 64, 2048),
            "weights": weights, "gated": rng.random() < 0.5, "type": weights if weights in TYPES else rng.choice(["bf16", "f16"])}


# ---- inputs --------------------------------------------------------------------------------------------------------------

def _up(n, unit):
    return -(-n // unit) * unit


def _activations(g, rows, cols, scale=1.0):
    x = torch.randn(rows, cols, generator=g, device="cuda") * scale
    x[:, torch.randint(0, cols, (max(1, cols // 256),), generator=g, device="cuda")] *= 12.0    # a few channels are large in every row
    return x


def _offsets(g, rows, experts):
    """First row of each expert: uneven, some of them empty."""
    p = torch.randn(experts, generator=g, device="cuda").mul(0.8).exp()
    p[torch.randint(0, experts, (max(1, experts // 16),), generator=g, device="cuda")] = 0.0
    counts = torch.bincount(torch.multinomial(p, rows, replacement=True, generator=g), minlength=experts)
    offsets = torch.zeros(experts + 1, dtype=torch.int64, device="cuda")
    offsets[1:] = torch.cumsum(counts, 0)
    return offsets


def _padded_room(rows, experts):
    return _up(rows + (GROUP - 1) * experts, GROUP)


def _padded_rows(offsets, rows):
    """Where each row lies if each expert's rows start at a multiple of 128."""
    padded = (offsets[1:] - offsets[:-1] + GROUP - 1) // GROUP * GROUP
    row = torch.arange(rows, device=offsets.device)
    expert = torch.searchsorted(offsets[1:].contiguous(), row, right=True)
    return (torch.cumsum(padded, 0) - padded)[expert] + row - offsets[:-1][expert]


def _spread_rows(x, offsets):
    """The rows of x at their places of _padded_rows, zeros between them."""
    room = _padded_room(x.shape[0], offsets.shape[0] - 1)
    return torch.zeros(room, x.shape[1], dtype=x.dtype, device="cuda").index_copy_(0, _padded_rows(offsets, x.shape[0]), x)


def _power_above(a, top):
    """Exponents k (biased by 127) of the smallest powers of two with a <= top * 2^k; a: fp32, top: 1.x * 2^n, exactly."""
    bits, t = a.view(torch.int32), torch.tensor(top, dtype=torch.float32, device=a.device).view(torch.int32)
    return (bits >> 23) - (t >> 23) + 127 + ((bits & 0x7FFFFF) > (t & 0x7FFFFF)).int()


def _factor(x, fmt):
    """The 32-bit factor of a tensor, or of each matrix of a stack."""
    if fmt != "nvfp4":
        return None
    amax = x.float().abs().amax((-2, -1)).reshape(-1)
    return torch.where(amax > 0, torch.ldexp(torch.ones_like(amax), _power_above(amax, 6.0 * FP8_MAX) - 127), 0.0)


def _operand(x, fmt, offsets=None):
    """x (..., R, C) as (bytes of two values each, scale tiles, factor)."""
    factor = _factor(x, fmt)
    codes, scales = _codes(x, fmt, factor)
    return _packed(codes), _tiles(scales if offsets is None else _spread_rows(scales, offsets)), factor


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 13)
    state = {"case": case}
    op = case["op"]
    if op == "quantize":
        R, C, top, experts, fmt = case["rows"], case["cols"], case["top"], case["experts"], case["format"]
        n, nb = R * max(1, top), BLOCK[fmt]
        state["x"] = _activations(g, R, C).to(TYPES[case["type"]])
        state["rows"] = state["offsets"] = None
        room = n
        if experts:
            state["rows"] = torch.randint(0, R, (n,), generator=g, device="cuda", dtype=torch.int32)
            state["offsets"] = _offsets(g, n, experts).to(torch.int32)
            room = _padded_room(n, experts)
        bytes_ = lambda *s: torch.zeros(*s, dtype=torch.uint8, device="cuda")  # noqa: E731
        atom = 4 * nb
        state["factor"] = torch.zeros(1, device="cuda")
        state["q"] = bytes_(n, _up(C, 32) // 2)[:, : (C + 1) // 2], bytes_(_up(room, GROUP) // GROUP, _up(C, atom) // atom, 512)
        state["values"] = torch.zeros(n, C, dtype=state["x"].dtype, device="cuda")
        if case["blocks"] == "both":
            state["q_cols"] = bytes_(C, _up(room, 32) // 2)[:, : (room + 1) // 2], bytes_(_up(C, GROUP) // GROUP, _up(room, atom) // atom, 512)
            state["values_cols"] = torch.zeros(C, room, dtype=state["x"].dtype, device="cuda")
    elif op in ("product", "experts"):
        form, N, K, fmt = case["form"], case["N"], case["K"], case["format"]
        experts = case["experts"] if op == "experts" else 0
        M = case["tokens"] * case["top"] if experts else case["M"]
        offsets = None
        if experts:
            offsets = _offsets(g, M, experts)
            state["most"] = int((offsets[1:] - offsets[:-1]).max())
            state["offsets"] = offsets.to(torch.int32)
        if form == "weight_grad":
            dy, x = torch.randn(M, N, generator=g, device="cuda") * 1e-3, _activations(g, M, K)
            if experts:
                dy, x = _spread_rows(dy, offsets), _spread_rows(x, offsets)
            state["a"], state["b"] = _operand(dy.t(), fmt), _operand(x.t(), fmt)
            shape = (experts, N, K) if experts else (N, K)
        else:
            a = _activations(g, M, K) if form == "forward" else torch.randn(M, N, generator=g, device="cuda") * 1e-3
            state["a"] = _operand(a, fmt, offsets)
            w = torch.randn(*((experts,) if experts else ()), N, K, generator=g, device="cuda") * K ** -0.5
            state["b"] = _operand(w if form == "forward" else w.transpose(-1, -2), fmt)
            shape = (M, N) if form == "forward" else (M, K)
        state["out"] = torch.zeros(*shape, dtype=TYPES[case["out"]], device="cuda")
        if own:
            from paper_2512_02551_b200 import fp4
            state["plan"] = fp4.Plan(_context(), M, N, K, form=form, groups=experts, format=fmt, out_dtype=TYPES[case["out"]])
    else:
        T, k, E, H, I = case["tokens"], case["top"], case["experts"], case["hidden"], case["inner"]
        dtype = TYPES[case["type"]]
        state["x"] = _activations(g, T, H).to(dtype)
        state["indices"] = torch.rand(T, E, generator=g, device="cuda").argsort(-1)[:, :k].int().contiguous()
        w = torch.rand(T, k, generator=g, device="cuda") + 0.1
        state["weights"] = w / w.sum(-1, keepdim=True)
        for name, n, m in (("w1", I * (2 if case["gated"] else 1), H), ("w2", H, I)):
            w = torch.randn(E, n, m, generator=g, device="cuda") * m ** -0.5
            state[name] = w.to(dtype) if case["weights"] in TYPES else _operand(w, case["weights"])
        state["y"] = torch.zeros(T, H, dtype=dtype, device="cuda")
        state["most"] = int(torch.bincount(state["indices"].reshape(-1), minlength=E).max())
        if own:
            from paper_2512_02551_b200 import few_tokens
            state["layer"] = few_tokens.Layer(_context(), H, I, E, k, weights=case["weights"], activation="swiglu" if case["gated"] else "silu", dtype=dtype)
            state["scratch"] = state["layer"].empty_scratch(T)
    return state


_contexts = []


def _context():
    """The library's context, one for the process, as a program keeps it."""
    if not _contexts:
        from paper_2512_02551_b200 import hgemm
        _contexts.append(hgemm.Context(0))
    return _contexts[0]


# ---- one pass ------------------------------------------------------------------------------------------------------------

def run(state):
    case = state["case"]
    if not own:
        return {"quantize": _plain_quantize, "product": _plain_product, "experts": _plain_experts, "layer": _plain_layer}[case["op"]](state, case)
    if case["op"] == "quantize":
        return _own_quantize(state, case)
    if case["op"] == "layer":
        state["layer"].run(state["x"], state["w1"], state["w2"], state["indices"], state["weights"], state["y"], state["scratch"])
        return state["y"]
    (a, sa, fa), (b, sb, fb) = state["a"], state["b"]
    state["plan"].run(a, sa, b, sb, state["out"], a_factor=fa, b_factor=fb, offsets=state.get("offsets"))
    return state["out"]


def _own_quantize(state, case):
    from paper_2512_02551_b200 import fp4
    ctx, x, fmt, at = _context(), state["x"], case["format"], state["offsets"]
    factor = None
    if fmt == "nvfp4":
        factor = state["factor"]
        fp4.tensor_factor(ctx, x, factor)
    if case["blocks"] == "both":
        fp4.quantize_both(ctx, x, *state["q"], *state["q_cols"], factor=factor, format=fmt, rows=state["rows"], offsets=at)
    else:
        fp4.quantize_rows(ctx, x, *state["q"], factor=factor, format=fmt, rows=state["rows"], offsets=at)
    fp4.dequantize(ctx, *state["q"], state["values"], factor=factor, format=fmt, offsets=at)
    if case["blocks"] == "rows":
        return [state["values"]]
    fp4.dequantize(ctx, *state["q_cols"], state["values_cols"], factor=factor, format=fmt)
    return [state["values"], state["values_cols"]]


# ---- plain forms, 32 bits --------------------------------------------------------------------------------------------------

def _e4m3(v):
    """v >= 0 rounded to an e4m3 value, at most the largest."""
    return v.clamp(max=FP8_MAX).to(torch.float8_e4m3fn)


def _codes(x, fmt, factor):
    """x (..., R, C) as 4-bit codes (sign, magnitude 0 .. 7) and scale bytes (..., R, blocks)."""
    nb, C = BLOCK[fmt], x.shape[-1]
    b = torch.nn.functional.pad(x.float(), (0, _up(C, nb) - C))
    b = b.view(*b.shape[:-1], -1, nb)
    amax = b.abs().amax(-1)
    if fmt == "nvfp4":
        f = factor.view(*factor.shape, 1, 1) if x.dim() == 3 else factor
        g = torch.where(f >= TINY, torch.ones_like(f) / f, 0.0)
        scale = _e4m3(amax * g * torch.tensor(1.0 / 6.0, device=x.device))
        step = scale.float() * f
        scale = scale.view(torch.uint8)
    else:
        e = _power_above(amax, 6.0).clamp(0, 254)
        step = torch.ldexp(torch.ones_like(amax), e - 127)
        scale = e.to(torch.uint8)
    step = step.unsqueeze(-1)
    v = torch.where(step > 0, b / step, 0.0)
    m = v.abs()
    code = (m > 0.25).to(torch.uint8) + (m >= 0.75) + (m > 1.25) + (m >= 1.75) + (m > 2.5) + (m >= 3.5) + (m > 5.0)
    code = code + 8 * (v < 0).to(torch.uint8)
    return code.reshape(*x.shape[:-1], -1)[..., :C], scale


def _packed(codes):
    """Two codes to a byte, the first in the low half; rows start at multiples of 16 bytes."""
    C = codes.shape[-1]
    wide = torch.nn.functional.pad(codes, (0, _up(C, 32) - C))
    return (wide[..., 0::2] | (wide[..., 1::2] << 4)).contiguous()[..., : (C + 1) // 2]


def _tiles(scales):
    """Scale bytes (..., R, blocks) as tiles of 128 rows x 4 blocks, 512 bytes each: byte 16 (r % 32) + 4 (r / 32) + j of row r, block j."""
    R, B = scales.shape[-2:]
    s = torch.nn.functional.pad(scales, (0, _up(B, 4) - B, 0, _up(R, GROUP) - R))
    s = s.view(*s.shape[:-2], s.shape[-2] // GROUP, 4, 32, s.shape[-1] // 4, 4)
    n = s.dim() - 5
    return s.permute(*range(n), n, n + 3, n + 2, n + 1, n + 4).reshape(*s.shape[:n], s.shape[n], s.shape[n + 3], 512)


def _scales(tiles, R, B):
    """The scale bytes (..., R, B) of _tiles."""
    s = tiles.view(*tiles.shape[:-1], 32, 4, 4)
    n = s.dim() - 5
    s = s.permute(*range(n), n, n + 3, n + 2, n + 1, n + 4)
    return s.reshape(*s.shape[:n], s.shape[n] * GROUP, s.shape[n + 3] * 4)[..., :R, :B]


_E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0]


def _values_of(codes, scale, fmt, factor, dtype=torch.float32):
    """What codes (..., R, C) and scale bytes (..., R, blocks) stand for."""
    table = torch.tensor(_E2M1, dtype=dtype, device="cuda")
    if fmt == "nvfp4":
        s = scale.contiguous().view(torch.float8_e4m3fn).to(dtype)
        s = s * (factor.to(dtype).view(*factor.shape, 1, 1) if codes.dim() == 3 else factor.to(dtype))
    else:
        s = torch.ldexp(torch.ones_like(scale, dtype=dtype), scale.int() - 127)
    return table[codes.int()] * s.repeat_interleave(BLOCK[fmt], -1)[..., : codes.shape[-1]]


def _values(operand, C, fmt, offsets=None, dtype=torch.float32):
    """What an operand stands for: (..., R, C)."""
    q, tiles, factor = operand
    R = q.shape[-2]
    codes = torch.stack((q & 15, q >> 4), -1).view(*q.shape[:-1], -1)[..., :C]
    blocks = -(-C // BLOCK[fmt])
    if offsets is None:
        s = _scales(tiles, R, blocks)
    else:
        s = _scales(tiles, tiles.shape[0] * GROUP, blocks)[_padded_rows(offsets, R)]
    return _values_of(codes, s, fmt, factor, dtype)


def _plain_quantize(state, case):
    x, fmt = state["x"].float(), case["format"]
    factor = _factor(x, fmt)
    if state["rows"] is not None:
        x = x[state["rows"].long()]
    out = [_values_of(*_codes(x, fmt, factor), fmt, factor).to(state["x"].dtype)]
    if case["blocks"] == "both":
        if state["offsets"] is not None:
            x = _spread_rows(x, state["offsets"].long())
        x = x.t()
        out.append(_values_of(*_codes(x, fmt, factor), fmt, factor).to(state["x"].dtype))
    return out


def _contracted(case, rows):
    return {"forward": case["K"], "input_grad": case["N"], "weight_grad": rows}[case["form"]]


def _plain_product(state, case):
    C, fmt = _contracted(case, case["M"]), case["format"]
    return (_values(state["a"], C, fmt) @ _values(state["b"], C, fmt).t()).to(TYPES[case["out"]])


def _plain_experts(state, case):
    """Every expert's rows in a slab as high as the fullest expert's, then one batched product."""
    E, most, offsets, fmt = case["experts"], state["most"], state["offsets"].long(), case["format"]
    counts = offsets[1:] - offsets[:-1]
    place = torch.arange(most, device="cuda")
    held = (place < counts[:, None]).unsqueeze(-1)
    rows = case["tokens"] * case["top"]
    if case["form"] == "weight_grad":
        room = _padded_room(rows, E)
        padded = (counts + GROUP - 1) // GROUP * GROUP
        at = ((torch.cumsum(padded, 0) - padded)[:, None] + place).clamp(max=room - 1)
        dy = torch.where(held, _values(state["a"], room, fmt).t()[at], 0.0)
        x = torch.where(held, _values(state["b"], room, fmt).t()[at], 0.0)
        return torch.bmm(dy.transpose(1, 2), x).to(TYPES[case["out"]])
    C = _contracted(case, rows)
    at = (offsets[:-1, None] + place).clamp(max=rows - 1)
    slab = torch.where(held, _values(state["a"], C, fmt, offsets)[at], 0.0)
    out = torch.bmm(slab, _values(state["b"], C, fmt).transpose(1, 2))
    row = torch.arange(rows, device="cuda")
    expert = torch.searchsorted(offsets[1:].contiguous(), row, right=True)
    return out[expert, row - offsets[expert]].to(TYPES[case["out"]])


def _weight(state, case, name, C, dtype=torch.float32):
    return state[name].to(dtype) if case["weights"] in TYPES else _values(state[name], C, case["weights"], dtype=dtype)


def _plain_layer(state, case):
    """The choices of each expert in a slab as high as the fullest expert's, two batched products, and the weighted sum over a token's choices."""
    T, k, E, H, I = case["tokens"], case["top"], case["experts"], case["hidden"], case["inner"]
    flat = state["indices"].reshape(-1).long()
    order = torch.sort(flat, stable=True).indices
    ends = torch.cumsum((flat[:, None] == torch.arange(E, device="cuda")).sum(0), 0)
    starts = torch.cat([torch.zeros_like(ends[:1]), ends[:-1]])
    place = torch.arange(state["most"], device="cuda")
    choice = order[(starts[:, None] + place).clamp(max=T * k - 1)]
    slab = state["x"].float()[choice // k]
    h = torch.bmm(slab, _weight(state, case, "w1", H).transpose(1, 2))
    gate = h[..., :I]
    h = gate / (1.0 + torch.exp(-gate)) * (h[..., I:] if case["gated"] else 1.0)
    rows = torch.bmm(h, _weight(state, case, "w2", I).transpose(1, 2))
    place_of = torch.empty_like(order).scatter_(0, order, torch.arange(T * k, device="cuda")) - starts[flat]
    picked = rows[flat, place_of].view(T, k, H)
    return (picked * state["weights"].unsqueeze(-1)).sum(1).to(state["y"].dtype)


# ---- what a pass cannot do without -----------------------------------------------------------------------------------------

def _bytes4(rows, cols, fmt):
    return rows * ((cols + 1) // 2 + -(-cols // BLOCK[fmt]))


def work(case):
    size = {"bf16": 2, "f16": 2, "f32": 4}
    op = case["op"]
    if op == "quantize":
        R, C, fmt = case["rows"], case["cols"], case["format"]
        n = R * max(1, case["top"])
        made = _bytes4(n, C, fmt) + n * C * size[case["type"]]
        if case["blocks"] == "both":
            made += _bytes4(C, n, fmt) + n * C * size[case["type"]]
        return {"bytes": R * C * size[case["type"]] + made + (4 * n if case["top"] else 0), "flops": 3 * n * C}
    if op in ("product", "experts"):
        N, K, fmt, form = case["N"], case["K"], case["format"], case["form"]
        M = case["tokens"] * case["top"] if op == "experts" else case["M"]
        E = case["experts"] if op == "experts" else 1
        used = min(E, M)            # weight matrices that can have a row
        held = {"forward": _bytes4(M, K, fmt) + used * _bytes4(N, K, fmt) + M * N * size[case["out"]],
                "input_grad": _bytes4(M, N, fmt) + used * _bytes4(K, N, fmt) + M * K * size[case["out"]],
                "weight_grad": _bytes4(N, M, fmt) + _bytes4(K, M, fmt) + E * N * K * size[case["out"]]}[form]
        return {"bytes": held, "flops": 2 * M * N * K}
    T, k, H, I = case["tokens"], case["top"], case["hidden"], case["inner"]
    used = case["experts"] * (1.0 - (1.0 - k / case["experts"]) ** T)       # experts that some token chooses, on average
    up = I * (2 if case["gated"] else 1)
    each = (up * H + H * I) * size[case["weights"]] if case["weights"] in size else _bytes4(up, H, case["weights"]) + _bytes4(H, I, case["weights"])
    return {"bytes": used * each + 2 * T * H * size[case["type"]] + 8 * T * k, "flops": 2 * T * k * (up * H + H * I)}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------------------

def _nearest4(v):
    """v (64 bits) rounded to the nearest of the 4-bit values, ties to the even code."""
    m = v.abs().clamp(max=6.0)
    step = torch.where(m < 2.0, 0.5, torch.where(m < 4.0, 1.0, 2.0)).double()
    return torch.copysign(torch.round(m / step) * step, v)


def _nearest8(v):
    """v >= 0 (64 bits) rounded to the nearest e4m3 value, ties to the even one."""
    step = torch.ldexp(torch.ones_like(v), torch.clamp(torch.frexp(v).exponent - 1, min=-6) - 3)
    return (torch.round(v / step) * step).clamp(max=FP8_MAX)


def _exact_rows(x, fmt, largest):
    """The values of x (R x C, 64 bits) held in 4 bits with blocks along its rows."""
    R, C = x.shape
    nb = BLOCK[fmt]
    b = torch.nn.functional.pad(x, (0, _up(C, nb) - C)).unfold(1, nb, nb)
    amax = b.abs().amax(-1, keepdim=True)
    if fmt == "nvfp4":
        factor = 2.0 ** math.ceil(math.log2(max(float(largest), 1e-300) / (6.0 * FP8_MAX)))
        scale = _nearest8(amax / (6.0 * factor)) * factor if float(largest) > 0 else torch.zeros_like(amax)
    else:
        up = torch.ceil(torch.log2(torch.where(amax > 0, amax, 1.0) / 6.0))
        up = up + (torch.exp2(up) * 6.0 < amax).double() - (torch.exp2(up - 1) * 6.0 >= amax).double()     # however the logarithm rounds
        scale = torch.where(amax > 0, torch.exp2(up.clamp(min=-127)), 0.0)
    v = _nearest4(b / torch.where(scale > 0, scale, 1.0)) * scale
    return v.reshape(R, -1)[:, :C]


def exact(case, seed):
    state = prepare(case, seed)
    op = case["op"]
    if op == "quantize":
        x = state["x"].double()
        largest = x.abs().max()
        if state["rows"] is not None:
            x = x[state["rows"].long()]
        out = [_exact_rows(x, case["format"], largest)]
        if case["blocks"] == "both":
            if state["offsets"] is not None:
                x = _spread_rows(x, state["offsets"].long())
            out.append(_exact_rows(x.t().contiguous(), case["format"], largest))
        return out
    if op in ("product", "experts"):
        form, fmt = case["form"], case["format"]
        if op == "product":
            C = _contracted(case, case["M"])
            return _values(state["a"], C, fmt, dtype=torch.float64).matmul(_values(state["b"], C, fmt, dtype=torch.float64).t())
        rows, E, ends = case["tokens"] * case["top"], case["experts"], state["offsets"].tolist()
        if form == "weight_grad":
            room = _padded_room(rows, E)
            a, b = _values(state["a"], room, fmt, dtype=torch.float64), _values(state["b"], room, fmt, dtype=torch.float64)
            out, start = [], 0
            for e in range(E):
                n = ends[e + 1] - ends[e]
                out.append(a[:, start:start + n].matmul(b[:, start:start + n].t()))
                start += _up(n, GROUP)
            return torch.stack(out)
        C = _contracted(case, rows)
        a = _values(state["a"], C, fmt, state["offsets"].long(), dtype=torch.float64)
        of = lambda e: _values(tuple(None if t is None else t[e:e + 1] for t in state["b"]), C, fmt, dtype=torch.float64)[0]  # noqa: E731
        return torch.cat([a[ends[e]:ends[e + 1]].matmul(of(e).t()) for e in range(E)])
    T, k, E, H, I = case["tokens"], case["top"], case["experts"], case["hidden"], case["inner"]
    y = torch.zeros(T, H, dtype=torch.float64, device="cuda")
    x, weights = state["x"].double(), state["weights"].double()
    for e in range(E):
        t, j = torch.nonzero(state["indices"] == e, as_tuple=True)
        if not len(t):
            continue
        part = lambda name: state[name][e:e + 1] if case["weights"] in TYPES else tuple(None if v is None else v[e:e + 1] for v in state[name])  # noqa: E731
        one = {"w1": part("w1"), "w2": part("w2")}
        h = x[t].matmul(_weight(one, case, "w1", H, torch.float64)[0].t())
        h = torch.nn.functional.silu(h[:, :I]) * (h[:, I:] if case["gated"] else 1.0)
        y.index_add_(0, t, weights[t, j].unsqueeze(-1) * h.matmul(_weight(one, case, "w2", I, torch.float64)[0].t()))
    return y

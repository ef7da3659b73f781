"""Measured cases of the 8-bit products with block scales, their quantiser, the products over experts and the routing to them.

Four operators.  "quantize" turns activations, gradients or weights into 8-bit values with one scale for each block of 128;
"product" is a linear layer's forward product, its input gradient or its weight gradient on such operands; "experts" is the
same with rows sorted by expert and one weight matrix for each expert; "route" chooses each token's experts from the router's
logits, sorts the (token, choice) pairs by expert and, for training, gives the logits' gradient.

Inputs: activations are normal with a few large channels, weights normal / sqrt(inputs), gradients normal and small, router
logits normal with a spread of about two.  Sizes are powers of two from 64 to 16384 and odd numbers between them.
"""
import math

import torch

own = False

BLOCK = 128
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
FP8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
FP8_MAX = {"e4m3": 448.0, "e5m2": 57344.0}
TINY = 2.0 ** -100          # a block whose largest magnitude is below this counts as zero


# ---- cases ---------------------------------------------------------------------------------------------------------------

def listed():
    return [
        # quantize: one decoding batch's activations before a projection; latency counts
        {"name": "quantize rows 24x4096", "op": "quantize", "blocks": "rows", "rows": 24, "cols": 4096, "type": "bf16", "fp8": "e4m3", "pow2": False, "top": 0},
        # ... a training batch's activations, needed along rows (forward) and along columns (weight gradient); odd row count
        {"name": "quantize both 8191x4096", "op": "quantize", "blocks": "both", "rows": 8191, "cols": 4096, "type": "bf16", "fp8": "e4m3", "pow2": False, "top": 0},
        # ... tokens gathered into expert order and quantised on the way, scales as powers of two
        {"name": "quantize gather 4096x8x2048", "op": "quantize", "blocks": "rows", "rows": 4096, "cols": 2048, "type": "f16", "fp8": "e4m3", "pow2": True, "top": 8},
        # product: a projection while decoding a few sequences: the weights' bytes bound it
        {"name": "forward 7x8192x4096", "op": "product", "form": "forward", "M": 7, "N": 8192, "K": 4096, "out": "bf16", "grad": "e4m3"},
        # ... a prompt of 1000 tokens, result in the library's fp16
        {"name": "forward 1000x4096x4096", "op": "product", "form": "forward", "M": 1000, "N": 4096, "K": 4096, "out": "f16", "grad": "e4m3"},
        # ... the largest square of the benchmark's middle grid: the tensor cores bound it
        {"name": "forward 8192x8192x8192", "op": "product", "form": "forward", "M": 8192, "N": 8192, "K": 8192, "out": "bf16", "grad": "e4m3"},
        # ... training: gradient of the inputs, sizes off every tile
        {"name": "input_grad 4000x4096x2000", "op": "product", "form": "input_grad", "M": 4000, "N": 4096, "K": 2000, "out": "bf16", "grad": "e5m2"},
        # ... training: gradient of the weights, kept in 32 bits
        {"name": "weight_grad 8192x4096x4096", "op": "product", "form": "weight_grad", "M": 8192, "N": 4096, "K": 4096, "out": "f32", "grad": "e4m3"},
        # experts: decoding, 32 tokens of 8 choices over 64 experts: about four rows for each weight matrix
        {"name": "experts forward 32x8 of 64", "op": "experts", "form": "forward", "tokens": 32, "top": 8, "experts": 64, "N": 2048, "K": 2048, "out": "bf16", "grad": "e4m3"},
        # ... training: 8192 tokens of 4 choices over 32 experts, gradient of each expert's weights
        {"name": "experts weight_grad 8192x4 of 32", "op": "experts", "form": "weight_grad", "tokens": 8192, "top": 4, "experts": 32, "N": 2048, "K": 2048, "out": "bf16", "grad": "e4m3"},
        # route: decoding, sigmoid scores with the balancing bias, groups and renormalised weights
        {"name": "route 33 tokens of 256", "op": "route", "tokens": 33, "experts": 256, "top": 8, "score": "sigmoid", "bias": True, "groups": 8, "top_groups": 4,
         "group_score": "top2", "renormalize": True, "type": "f32", "backward": False},
        # ... training: softmax scores, forward and backward
        {"name": "route 16384 tokens of 128", "op": "route", "tokens": 16384, "experts": 128, "top": 8, "score": "softmax", "bias": False, "groups": 1, "top_groups": 1,
         "group_score": "max", "renormalize": True, "type": "bf16", "backward": True},
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["quantize", "product", "product", "experts", "experts", "route"])
    if op == "quantize":
        blocks = rng.choice(["rows", "both", "tiles"])
        top = rng.choice([0, 2, 4, 8]) if blocks == "rows" else 0
        cols = _log(rng, 64, 8192)
        rows = _log(rng, 1, min(16384, (8191 * 4096) // (cols * max(1, top))))
        return {"op": op, "blocks": blocks, "rows": rows, "cols": cols, "type": rng.choice(list(TYPES)), "fp8": rng.choice(list(FP8)), "pow2": rng.random() < 0.5, "top": top}
    if op == "product":
        form = rng.choice(["forward", "forward", "input_grad", "weight_grad"])
        return {"op": op, "form": form, "M": _log(rng, 1, 8192), "N": _log(rng, 64, 8192), "K": _log(rng, 64, 8192), "out": rng.choice(list(TYPES)),
                "grad": rng.choice(list(FP8)) if form != "forward" else "e4m3"}
    if op == "experts":
        form = rng.choice(["forward", "input_grad", "weight_grad"])
        experts = rng.choice([8, 16, 32, 48, 64])
        return {"op": op, "form": form, "tokens": _log(rng, 1, 8192), "top": rng.choice([1, 2, 4, 8]), "experts": experts, "N": _log(rng, 64, 2048),
                "K": _log(rng, 64, 2048), "out": rng.choice(list(TYPES)), "grad": rng.choice(list(FP8)) if form != "forward" else "e4m3"}
    experts = rng.choice([8, 16, 60, 64, 128, 160, 256, 512])
    score = rng.choice(["softmax", "sigmoid"])
    groups = rng.choice([1, 1, 4]) if experts >= 60 else 1
    return {"op": op, "tokens": _log(rng, 1, 16384), "experts": experts, "top": rng.choice([1, 2, 4, 6, 8]), "score": score, "bias": score == "sigmoid" and rng.random() < 0.6,
            "groups": groups, "top_groups": 2 if groups > 1 else 1, "group_score": "top2" if score == "sigmoid" and groups > 1 else "max",
            "renormalize": rng.random() < 0.6, "type": rng.choice(list(TYPES)), "backward": rng.random() < 0.5}


# ---- inputs --------------------------------------------------------------------------------------------------------------

def _up(n, unit):
    return -(-n // unit) * unit


def _pitched(q):
    """8-bit rows start at multiples of 16 bytes, as the products need them: a view of a wider tensor where they would not."""
    wide = torch.zeros(*q.shape[:-1], _up(q.shape[-1], 16), dtype=q.dtype, device=q.device)
    wide[..., : q.shape[-1]] = q
    return wide[..., : q.shape[-1]]


def _activations(g, rows, cols, scale=1.0):
    x = torch.randn(rows, cols, generator=g, device="cuda") * scale
    x[:, torch.randint(0, cols, (max(1, cols // 256),), generator=g, device="cuda")] *= 12.0    # a few channels are large in every row
    return x


def _counts(g, rows, experts):
    """Rows of each expert: uneven, some of them empty."""
    p = torch.randn(experts, generator=g, device="cuda").mul(0.8).exp()
    p[torch.randint(0, experts, (max(1, experts // 16),), generator=g, device="cuda")] = 0.0
    picked = torch.multinomial(p, rows, replacement=True, generator=g)
    return torch.bincount(picked, minlength=experts)


def _padded_rows(offsets, rows, experts):
    """The row of the padded copy, in which each expert's rows start at a multiple of 128, of every row."""
    counts = offsets[1:] - offsets[:-1]
    starts = torch.cumsum((counts + BLOCK - 1) // BLOCK * BLOCK, 0) - (counts + BLOCK - 1) // BLOCK * BLOCK
    row = torch.arange(rows, device=offsets.device)
    expert = torch.searchsorted(offsets[1:].contiguous(), row, right=True)
    return starts[expert] + row - offsets[:-1][expert]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 13)
    state = {"case": case}
    op = case["op"]
    if op == "quantize":
        R, C, top = case["rows"], case["cols"], case["top"]
        x = (_activations(g, R, C) if case["blocks"] != "tiles" else torch.randn(R, C, generator=g, device="cuda") * C ** -0.5).to(TYPES[case["type"]])
        out_rows = R * top if top else R
        f8 = FP8[case["fp8"]]
        state["x"] = x
        state["rows"] = torch.randint(0, R, (out_rows,), generator=g, device="cuda", dtype=torch.int32) if top else None
        if case["blocks"] == "tiles":
            state["out"] = [_pitched(torch.zeros(R, C, dtype=f8, device="cuda")), torch.zeros(_up(R, BLOCK) // BLOCK, _up(C, BLOCK) // BLOCK, device="cuda")]
        else:
            state["out"] = [_pitched(torch.zeros(out_rows, C, dtype=f8, device="cuda")), torch.zeros(out_rows, _up(C, BLOCK) // BLOCK, device="cuda")]
            if case["blocks"] == "both":
                state["out"] += [_pitched(torch.zeros(R, C, dtype=f8, device="cuda")), torch.zeros(_up(R, BLOCK) // BLOCK, C, device="cuda")]
    elif op in ("product", "experts"):
        form, N, K = case["form"], case["N"], case["K"]
        experts = case["experts"] if op == "experts" else 0
        M = case["tokens"] * case["top"] if experts else case["M"]
        offsets = None
        if experts:
            offsets = torch.zeros(experts + 1, dtype=torch.int64, device="cuda")
            counts = _counts(g, M, experts)
            offsets[1:] = torch.cumsum(counts, 0)
            state["most"] = int(counts.max())
            state["offsets"] = offsets.to(torch.int32)
        if form == "weight_grad":
            dy, x = torch.randn(M, N, generator=g, device="cuda") * 1e-3, _activations(g, M, K)
            if experts:             # each expert's rows start at a multiple of 128 of the quantised copy, zeros between them
                at = _padded_rows(offsets, M, experts)
                room = _up(M + 127 * experts, BLOCK)
                dy = torch.zeros(room, N, device="cuda").index_copy_(0, at, dy)
                x = torch.zeros(room, K, device="cuda").index_copy_(0, at, x)
            state["a"], state["sa"] = _quantize(dy, "cols", case["grad"], False)
            state["b"], state["sb"] = _quantize(x, "cols", "e4m3", False)
            shape = (experts, N, K) if experts else (N, K)
        else:
            a = _activations(g, M, K) if form == "forward" else torch.randn(M, N, generator=g, device="cuda") * 1e-3
            state["a"], state["sa"] = _quantize(a, "rows", case["grad"], False)
            w = torch.randn(max(1, experts), N, K, generator=g, device="cuda") * K ** -0.5
            w8, sw = _quantize(w, "tiles", "e4m3", False)
            state["b"], state["sb"] = (w8, sw) if experts else (w8[0], sw[0])
            shape = (M, N) if form == "forward" else (M, K)
        state["a"], state["b"] = _pitched(state["a"]), _pitched(state["b"])
        state["out"] = torch.zeros(*shape, dtype=TYPES[case["out"]], device="cuda")
        if own:
            from paper_2512_02551_b200 import fp8
            state["plan"] = fp8.Plan(_context(), M, N, K, form=case["form"], groups=experts, a_dtype=FP8[case["grad"]], b_dtype=FP8["e4m3"], out_dtype=TYPES[case["out"]])
    else:
        T, E, k = case["tokens"], case["experts"], case["top"]
        state["logits"] = (torch.randn(T, E, generator=g, device="cuda") * 2.0).to(TYPES[case["type"]])
        state["bias"] = torch.randn(E, generator=g, device="cuda") * 0.1 if case["bias"] else None
        state["dweights"] = torch.randn(T, k, generator=g, device="cuda") if case["backward"] else None
        state["out"] = [torch.zeros(T, k, device="cuda"), torch.zeros(T, k, dtype=torch.int32, device="cuda"), torch.zeros(E + 1, dtype=torch.int32, device="cuda"),
                        torch.zeros(T * k, dtype=torch.int32, device="cuda"), torch.zeros(T * k, dtype=torch.int32, device="cuda")]
        if case["backward"]:
            state["out"].append(torch.zeros(T, E, dtype=TYPES[case["type"]], device="cuda"))
        if own:
            from paper_2512_02551_b200 import routing
            state["router"] = routing.Router(_context(), E, k, score=case["score"], groups=case["groups"], top_groups=case["top_groups"], group_score=case["group_score"],
                                             renormalize=case["renormalize"], scale=1.0)
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
        return {"quantize": _plain_quantize, "product": _plain_product, "experts": _plain_experts, "route": _plain_route}[case["op"]](state, case)
    out = state["out"]
    if case["op"] == "quantize":
        from paper_2512_02551_b200 import fp8
        if case["blocks"] == "rows":
            fp8.quantize_rows(_context(), state["x"], out[0], out[1], rows=state["rows"], pow2=case["pow2"])
        elif case["blocks"] == "both":
            fp8.quantize_both(_context(), state["x"], out[0], out[1], out[2], out[3], pow2=case["pow2"])
        else:
            fp8.quantize_tiles(_context(), state["x"], out[0], out[1], pow2=case["pow2"])
    elif case["op"] == "product":
        state["plan"].run(state["a"], state["sa"], state["b"], state["sb"], out)
    elif case["op"] == "experts":
        state["plan"].run(state["a"], state["sa"], state["b"], state["sb"], out, offsets=state["offsets"])
    else:
        router = state["router"]
        router.forward(state["logits"], out[0], out[1], bias=state["bias"])
        router.sort(out[1], out[2], out[3], out[4])
        if case["backward"]:
            router.backward(state["logits"], out[1], state["dweights"], out[5])
    return out


# ---- plain forms, 32 bits --------------------------------------------------------------------------------------------------

def _blocks(x, rows, cols):
    """x (..., R, C) as (..., R / rows, rows, C / cols, cols), with zeros beyond the edges."""
    R, C = x.shape[-2:]
    x = torch.nn.functional.pad(x, (0, _up(C, cols) - C, 0, _up(R, rows) - R))
    return x.reshape(*x.shape[:-2], x.shape[-2] // rows, rows, x.shape[-1] // cols, cols)


def _quantize(x, blocks, fp8, pow2):
    """8-bit values and scales of x (..., R, C) in blocks of 1 x 128 ("rows"), 128 x 1 ("cols") or 128 x 128 ("tiles")."""
    R, C = x.shape[-2:]
    b = _blocks(x.float(), 1 if blocks == "rows" else BLOCK, 1 if blocks == "cols" else BLOCK)
    amax = torch.where(torch.isfinite(b), b.abs(), 0.0).amax((-3, -1), keepdim=True)
    some = amax >= TINY
    safe = torch.where(some, amax, 1.0)
    if pow2:
        mantissa, exponent = torch.frexp(safe / FP8_MAX[fp8])
        exponent = exponent - (mantissa == 0.5).int()
        scale, factor = torch.ldexp(torch.ones_like(safe), exponent), torch.ldexp(torch.ones_like(safe), -exponent)
    else:
        scale, factor = safe / FP8_MAX[fp8], FP8_MAX[fp8] / safe
    scale = torch.where(some, scale, 1.0)
    v = torch.where(some, b * factor, b * 0.0)
    v = torch.where(torch.isfinite(b), v.clamp(-FP8_MAX[fp8], FP8_MAX[fp8]), math.nan)
    v = v.reshape(*v.shape[:-4], v.shape[-4] * v.shape[-3], v.shape[-2] * v.shape[-1])[..., :R, :C]
    return v.to(FP8[fp8]), scale.squeeze(-1).squeeze(-2).contiguous()


def _values(q, s, blocks):
    """What 8-bit values and their scales stand for, in 32 bits."""
    R, C = q.shape[-2:]
    if blocks != "rows":
        s = s.repeat_interleave(BLOCK, -2)[..., :R, :]
    if blocks != "cols":
        s = s.repeat_interleave(BLOCK, -1)[..., :C]
    return q.float() * s


def _plain_quantize(state, case):
    x = state["x"].float()
    if state["rows"] is not None:
        x = x[state["rows"].long()]
    if case["blocks"] != "both":
        return list(_quantize(x, case["blocks"], case["fp8"], case["pow2"]))
    return [*_quantize(x, "rows", case["fp8"], case["pow2"]), *_quantize(x, "cols", case["fp8"], case["pow2"])]


def _plain_product(state, case):
    if case["form"] == "weight_grad":
        out = _values(state["a"], state["sa"], "cols").t() @ _values(state["b"], state["sb"], "cols")
    else:
        w = _values(state["b"], state["sb"], "tiles")
        out = _values(state["a"], state["sa"], "rows") @ (w.t() if case["form"] == "forward" else w)
    return out.to(TYPES[case["out"]])


def _plain_experts(state, case):
    """Every expert's rows in a slab as high as the fullest expert's, then one batched product."""
    E, most, offsets = case["experts"], state["most"], state["offsets"].long()
    counts = offsets[1:] - offsets[:-1]
    place = torch.arange(most, device="cuda")
    held = (place < counts[:, None]).unsqueeze(-1)
    rows = case["tokens"] * case["top"]
    if case["form"] == "weight_grad":
        padded = (counts + BLOCK - 1) // BLOCK * BLOCK
        at = ((torch.cumsum(padded, 0) - padded)[:, None] + place).clamp(max=state["a"].shape[0] - 1)
        dy = torch.where(held, _values(state["a"], state["sa"], "cols")[at], 0.0)
        x = torch.where(held, _values(state["b"], state["sb"], "cols")[at], 0.0)
        return torch.bmm(dy.transpose(1, 2), x).to(TYPES[case["out"]])
    at = (offsets[:-1, None] + place).clamp(max=rows - 1)
    slab = torch.where(held, _values(state["a"], state["sa"], "rows")[at], 0.0)
    w = _values(state["b"], state["sb"], "tiles")
    out = torch.bmm(slab, w.transpose(1, 2) if case["form"] == "forward" else w)
    row = torch.arange(rows, device="cuda")
    expert = torch.searchsorted(offsets[1:].contiguous(), row, right=True)
    return out[expert, row - offsets[expert]].to(TYPES[case["out"]])


def _plain_route(state, case):
    T, E, k, G = case["tokens"], case["experts"], case["top"], case["groups"]
    l = state["logits"].float()
    if case["score"] == "sigmoid":
        s = 1.0 / (1.0 + torch.exp(-l))
    else:
        e = torch.exp(l - l.amax(-1, keepdim=True))
        s = e / e.sum(-1, keepdim=True)
    v = s + state["bias"] if state["bias"] is not None else l if case["score"] == "softmax" else s
    if G > 1:
        grouped = v.view(T, G, E // G)
        if case["group_score"] == "top2":
            first_two = torch.sort(grouped, dim=-1, descending=True).values[..., :2]
            of_group = first_two[..., 0] + first_two[..., 1]
        else:
            of_group = grouped.amax(-1)
        kept = torch.sort(of_group, dim=-1, descending=True, stable=True).indices[:, : case["top_groups"]]
        keep = torch.zeros(T, G, dtype=torch.bool, device="cuda").scatter_(1, kept, True)
        v = torch.where(keep.unsqueeze(-1), grouped, -math.inf).view(T, E)
    indices = torch.sort(v, dim=-1, descending=True, stable=True).indices[:, :k]
    chosen = s.gather(1, indices)
    total = chosen.sum(-1, keepdim=True) + 1e-20
    weights = chosen / total if case["renormalize"] else chosen
    flat = indices.reshape(-1)
    order = torch.sort(flat, stable=True).indices
    offsets = torch.zeros(E + 1, dtype=torch.int64, device="cuda")
    offsets[1:] = torch.cumsum((flat[:, None] == torch.arange(E, device="cuda")).sum(0), 0)
    position = torch.empty_like(order).scatter_(0, order, torch.arange(T * k, device="cuda"))
    out = [weights, indices.int(), offsets.int(), order.int(), position.int()]
    if case["backward"]:
        dw = state["dweights"]
        d = (dw - (dw * weights).sum(-1, keepdim=True)) / total if case["renormalize"] else dw
        ds = torch.zeros_like(s).scatter_(1, indices, d)
        dl = ds * s * (1.0 - s) if case["score"] == "sigmoid" else s * (ds - (s * ds).sum(-1, keepdim=True))
        out.append(dl.to(TYPES[case["type"]]))
    return out


# ---- what a pass cannot do without -----------------------------------------------------------------------------------------

def work(case):
    size = {"bf16": 2, "f16": 2, "f32": 4}
    if case["op"] == "quantize":
        R, C = case["rows"], case["cols"]
        rows = R * case["top"] if case["top"] else R
        made = {"rows": rows * C + 4 * rows * (_up(C, BLOCK) // BLOCK), "tiles": R * C + 4 * (_up(R, BLOCK) // BLOCK) * (_up(C, BLOCK) // BLOCK),
                "both": 2 * R * C + 4 * R * (_up(C, BLOCK) // BLOCK) + 4 * C * (_up(R, BLOCK) // BLOCK)}[case["blocks"]]
        return {"bytes": R * C * size[case["type"]] + (4 * rows if case["top"] else 0) + made, "flops": 3 * rows * C}
    if case["op"] == "product":
        M, N, K = case["M"], case["N"], case["K"]
        held = {"forward": (M * K, N * K, M * N), "input_grad": (M * N, N * K, M * K), "weight_grad": (M * N, M * K, N * K)}[case["form"]]
        return {"bytes": held[0] + held[1] + held[2] * size[case["out"]] + 4 * (held[0] + held[1]) // BLOCK, "flops": 2 * M * N * K}
    if case["op"] == "experts":
        rows, N, K, E = case["tokens"] * case["top"], case["N"], case["K"], case["experts"]
        used = min(E, rows)         # weight matrices that can have a row
        held = {"forward": (rows * K, used * N * K, rows * N), "input_grad": (rows * N, used * N * K, rows * K), "weight_grad": (rows * N, rows * K, E * N * K)}[case["form"]]
        return {"bytes": held[0] + held[1] + held[2] * size[case["out"]] + 4 * (E + 1), "flops": 2 * rows * N * K}
    T, E, k = case["tokens"], case["experts"], case["top"]
    return {"bytes": T * E * size[case["type"]] * (3 if case["backward"] else 1) + T * k * (16 + (8 if case["backward"] else 0)) + 4 * (E + 1), "flops": T * E * (12 if case["backward"] else 6)}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------------------

def _spread(s, rows, cols, R, C):
    """Scales in 64 bits, one for each element of an R x C matrix whose blocks are rows x cols."""
    i, j = torch.arange(R, device="cuda") // rows, torch.arange(C, device="cuda") // cols
    return s.double()[..., i, :][..., j]


def _nearest8(v, fp8):
    """v (64 bits) rounded to the nearest value that the 8-bit type holds, ties to the even one."""
    bits, least = (3, -6) if fp8 == "e4m3" else (2, -14)
    exponent = torch.frexp(v).exponent - 1
    step = torch.ldexp(torch.ones_like(v), torch.clamp(exponent, min=least) - bits)
    return torch.round(v / step) * step


def _exact_quantize(x, rows, cols, case):
    R, C = x.shape
    top = FP8_MAX[case["fp8"]]
    down = torch.nn.functional.pad(x.abs(), (0, _up(C, cols) - C, 0, _up(R, rows) - R))
    largest = down.unfold(0, rows, rows).unfold(1, cols, cols).amax((-2, -1))
    scale = largest / top
    if case["pow2"]:
        below = torch.exp2(torch.floor(torch.log2(torch.where(largest > 0, scale, 1.0))) - 1)     # a power of two at most the scale, however the logarithm rounds
        scale = below * torch.exp2((below < scale).double() + (2 * below < scale).double() + (4 * below < scale).double())
    scale = torch.where(largest >= TINY, scale, 1.0)
    return [_nearest8(x / _spread(scale, rows, cols, R, C), case["fp8"]), scale]


def exact(case, seed):
    state = prepare(case, seed)
    op = case["op"]
    if op == "quantize":
        x = state["x"].double()
        x = x if state["rows"] is None else x[state["rows"].long()]
        if case["blocks"] == "tiles":
            return _exact_quantize(x, BLOCK, BLOCK, case)
        by_rows = _exact_quantize(x, 1, BLOCK, case)
        return by_rows if case["blocks"] == "rows" else by_rows + _exact_quantize(x, BLOCK, 1, case)
    if op in ("product", "experts"):
        a, b = state["a"].double(), state["b"].double()
        if case["form"] == "weight_grad":
            a, b = a * _spread(state["sa"], BLOCK, 1, *a.shape), b * _spread(state["sb"], BLOCK, 1, *b.shape)
            if op == "product":
                return a.t().matmul(b)
            ends, out, start = state["offsets"].tolist(), [], 0
            for e in range(case["experts"]):
                n = ends[e + 1] - ends[e]
                out.append(a[start:start + n].t().matmul(b[start:start + n]))
                start += _up(n, BLOCK)
            return torch.stack(out)
        a = a * _spread(state["sa"], 1, BLOCK, *a.shape)
        b = b * _spread(state["sb"], BLOCK, BLOCK, *b.shape[-2:])
        turn = (lambda w: w.t()) if case["form"] == "forward" else (lambda w: w)
        if op == "product":
            return a.matmul(turn(b))
        ends = state["offsets"].tolist()
        return torch.cat([a[ends[e]:ends[e + 1]].matmul(turn(b[e])) for e in range(case["experts"])])
    T, E, k = case["tokens"], case["experts"], case["top"]
    l = state["logits"].double()
    s = torch.sigmoid(l) if case["score"] == "sigmoid" else torch.softmax(l, -1)
    v = s if state["bias"] is None else s + state["bias"].double()
    if case["groups"] > 1:
        of = v.view(T, case["groups"], -1)
        rank = of.topk(2, -1).values.sum(-1) if case["group_score"] == "top2" else of.max(-1).values
        out_of = torch.ones_like(rank, dtype=torch.bool).scatter(1, rank.topk(case["top_groups"], -1).indices, False)
        v = of.masked_fill(out_of.unsqueeze(-1), -math.inf).view(T, E)
    # bf16 and fp16 logits tie often; the chosen weights are the same whichever of them is taken
    pick = torch.argsort(v, dim=-1, descending=True, stable=True)[:, :k]
    l = l.requires_grad_(case["backward"])
    s = torch.sigmoid(l) if case["score"] == "sigmoid" else torch.softmax(l, -1)
    w = s.gather(1, pick)
    w = w / (w.sum(-1, keepdim=True) + 1e-20) if case["renormalize"] else w
    out = [w.detach(), None, None, None, None]
    if case["backward"]:
        out.append(torch.autograd.grad((w * state["dweights"].double()).sum(), l)[0])
    return out

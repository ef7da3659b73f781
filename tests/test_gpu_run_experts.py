"""The layer of experts on 4-bit operands and its decoding step: the operators as ``run_experts`` puts them together."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2512_02551_b200 import fp4, hgemm  # noqa: E402
from paper_2512_02551_b200.run_experts import ExpertLayer  # noqa: E402

T, H, I, E, K = 300, 256, 192, 6, 2


@pytest.fixture(scope="module")
def ctx():
    assert torch.cuda.is_available(), "these tests need a B200"
    with hgemm.Context(0) as c:
        yield c


def inputs():
    g = torch.Generator(device="cuda").manual_seed(11)
    return torch.randn(T, H, generator=g, device="cuda").half(), torch.randn(T, H, generator=g, device="cuda")


def near(a, b):
    return float((a.double() - b.detach()).norm() / b.detach().norm())


def exact_layer(layer, x, indices, w1, w2):
    """The layer in 64 bits, the choice taken as it was made."""
    p = torch.softmax(x @ layer.wr.double().t(), -1).gather(1, indices.long())
    p = p / p.sum(-1, keepdim=True)
    y = torch.zeros_like(x)
    for e in range(layer.E):
        t, j = torch.nonzero(indices == e, as_tuple=True)
        y = y.index_add(0, t, p[t, j].unsqueeze(-1) * (torch.nn.functional.silu(x[t] @ w1[e].t()) @ w2[e].t()))
    return y


@pytest.mark.parametrize("operands", ["nvfp4", "mxfp4"])
def test_training_step(ctx, operands):
    """Against the same layer in 64 bits without quantisation: an element of a 4-bit copy is within 2^-2 of itself, or of its block's least step, so a
    quantised operand is within 2^-2 / sqrt(3) of the operand's norm for spread-out mantissas; at most four stand between input and output.  Then every
    product against the same product in 64 bits of what its copies stand for: fp32 sums over at most 300 terms and one rounding to bf16
    (2^-8 of each element at most)."""
    x, dy = inputs()
    with ExpertLayer(ctx, T, H, I, E, K, seed=5, operands=operands) as layer:
        y = layer.forward(x)
        dx, dw1, dw2, dlogits = layer.backward(dy)
        assert ctx.last_device_status()[0] == hgemm.OK
        xd, w1, w2 = x.double().requires_grad_(), layer.w1.double().requires_grad_(), layer.w2.double().requires_grad_()
        want = exact_layer(layer, xd, layer.indices, w1, w2)
        want.backward(dy.double())
        bound = 4 * 2.0 ** -2 / 3 ** 0.5
        for got, exact in ((y, want), (dx, xd.grad), (dw1, w1.grad), (dw2, w2.grad)):
            assert near(got, exact) < bound

        def stands(copies, n):
            out = torch.empty(T * K, n, device="cuda")
            fp4.dequantize(ctx, *copies.rows, out, factor=copies.factor, format=operands, offsets=layer.offsets)
            return out.double()

        def weights(w, by_columns):
            shape = w.rows[0].shape[0], *((I, H) if w is layer.q1 else (H, I))
            out = torch.empty(shape[0], *(shape[:0:-1] if by_columns else shape[1:]), device="cuda")
            fp4.dequantize(ctx, *(w.cols if by_columns else w.rows), out, factor=w.factor, format=operands)
            return out.double()

        def columns(copies, n):
            """What the column copy stands for, each expert's places, as rows."""
            v, s = copies.cols
            out = torch.empty(n, v.shape[1] * 2, device="cuda")
            fp4.dequantize(ctx, v, s, out, factor=copies.factor, format=operands)
            return out.double().t()

        offsets, at, places = layer.offsets.tolist(), 0, []
        for e in range(E):
            places.append(slice(at, at + offsets[e + 1] - offsets[e]))
            at += -(-(offsets[e + 1] - offsets[e]) // 128) * 128
        xs, a, dys, dh = stands(layer.xq, H), stands(layer.aq, I), stands(layer.dyq, H), stands(layer.dhq, I)
        f1, f2, b1, b2 = weights(layer.q1, False), weights(layer.q2, False), weights(layer.q1, True), weights(layer.q2, True)
        xc, ac, dyc, dhc = (columns(c, n) for c, n in ((layer.xq, H), (layer.aq, I), (layer.dyq, H), (layer.dhq, I)))
        for e in range(E):
            r, c = slice(offsets[e], offsets[e + 1]), places[e]
            if r.start == r.stop:
                continue
            for got, p, q in ((layer.h[r], xs[r], f1[e].t()), (layer.y_rows[r], a[r], f2[e].t()), (layer.da[r], dys[r], b2[e].t()), (layer.dx_rows[r], dh[r], b1[e].t()),
                              (dw1[e], dhc[c].t(), xc[c]), (dw2[e], dyc[c].t(), ac[c])):
                assert near(got, p @ q) < 2.0 ** -8, e


@pytest.mark.parametrize("operands,t", [("nvfp4", 1), ("nvfp4", 17), ("nvfp4", 64), ("mxfp4", 5), ("fp8", 1), ("fp8", 9)])
def test_decoding_step(ctx, operands, t):
    """Decoding steps against the layer in 64 bits with the weights that the step reads: x and h at 16 bits of mantissa or more, the router's logits and
    y in fp16 (a logit below 8 is off by 2^-9 at most, so a weight by 2^-8 of itself).  A training step in between changes nothing, a change of the
    weights is seen after ``refresh_weights``."""
    x, dy = inputs()
    with ExpertLayer(ctx, T, H, I, E, K, seed=5, operands=operands) as layer:
        for scale in (1.0, -0.5):
            layer.w1.mul_(scale)
            layer.refresh_weights()
            y = layer.decode(x[:t])
            layer.forward(x)
            layer.backward(dy)
            again = layer.decode(x[:t])
            assert torch.equal(y, again)
            if operands == "fp8":
                w1, w2 = layer.w1.half().double(), layer.w2.half().double()
            else:
                w1, w2 = torch.empty(E, I, H, device="cuda"), torch.empty(E, H, I, device="cuda")
                for w, q in ((w1, layer.q1), (w2, layer.q2)):
                    fp4.dequantize(ctx, *q.rows, w, factor=q.factor, format=operands)
                w1, w2 = w1.double(), w2.double()
            want = exact_layer(layer, x[:t].double(), layer.indices[:t], w1, w2)
            assert near(y, want) < 2.0 ** -7
        assert ctx.last_device_status()[0] == hgemm.OK


def test_decoding_steps_captured(ctx):
    """Two layers' steps in one graph, replayed with other tokens."""
    x, _ = inputs()
    with ExpertLayer(ctx, T, H, I, E, K, seed=1, operands="nvfp4") as one, ExpertLayer(ctx, T, H, I, E, K, seed=2, operands="mxfp4") as two:
        xs = x[:3].clone()
        two.decode(one.decode(xs))
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = two.decode(one.decode(xs))
        for i in (0, 7, 100):
            xs.copy_(x[i:i + 3])
            graph.replay()
            assert torch.equal(out, two.decode(one.decode(xs)))
        assert ctx.last_device_status()[0] == hgemm.OK


def test_refusals(ctx):
    with pytest.raises(ValueError):
        ExpertLayer(ctx, 8, 128, 128, 2, 1, operands="int4")
    with ExpertLayer(ctx, 8, 128, 128, 2, 1, operands="nvfp4") as layer:
        with pytest.raises(ValueError):
            layer.decode(torch.zeros(65, 128, dtype=torch.float16, device="cuda"))
        assert layer.decode(torch.zeros(0, 128, dtype=torch.float16, device="cuda")).shape == (0, 128)


def test_eight_bit_copies_by_their_names(ctx):
    """The 8-bit copies and the weights' tiles as a program hands them to products of its own."""
    x, dy = inputs()
    with ExpertLayer(ctx, T, H, I, E, K, seed=5) as layer:
        layer.forward(x)
        layer.backward(dy)
        h, dx_rows, dw2 = torch.empty_like(layer.h), torch.empty_like(layer.dx_rows), torch.empty_like(layer.dw2)
        layer.up.run(*layer.x8, *layer.q1, h, offsets=layer.offsets)
        layer.up_dx.run(*layer.dh8, *layer.q1, dx_rows, offsets=layer.offsets)
        layer.down_dw.run(*layer.dy8c, *layer.a8c, dw2, offsets=layer.offsets)
        assert torch.equal(h, layer.h) and torch.equal(dx_rows, layer.dx_rows) and torch.equal(dw2, layer.dw2)
        values, scales = layer.q2
        assert len(layer.q2) == 2 and layer.q2[0] is values and values.shape == (E, H, I)
        assert all(len(c) == 2 for c in (layer.a8, layer.dy8, layer.x8c, layer.dh8c))

"""One training step of a layer of experts on the 8-bit or the 4-bit products, end to end, and a decoding step with its weights; their device times.

    python -m paper_2512_02551_b200.run_experts [--tokens 4096] [--hidden 2048] [--inner 1024] [--experts 32] [--top-k 4] [--iters 5]
                                                [--operands fp8|nvfp4|mxfp4] [--decode 16]

``ExpertLayer`` shows how the pieces fit: the router's logits are a half-precision product (``hgemm``), the routing chooses
and orders (``routing``), tokens are gathered into expert order and quantised in one pass (``fp8.quantize_*``), each expert's two
products run as one grouped launch (``fp8.Plan`` with groups), and the backward pass uses the same weights' tiles for the
input gradients and column copies laid out per expert for the weight gradients.  With operands="nvfp4" or "mxfp4" the products are
those of ``fp4``: every operand has a row copy and a column copy (the input gradients take the weights' column copies) and, for "nvfp4", the
tensor's factor.  ``decode`` runs the layer on a few tokens (``few_tokens``) with the 4-bit weights, or with half-precision ones
beside 8-bit operands.
"""
from __future__ import annotations

import argparse

import torch

from . import few_tokens, fp4, fp8, hgemm, routing

OPERANDS = ("fp8", "nvfp4", "mxfp4")


class _Copies:
    """Room for an activation's row copy and column copy laid out per expert, and for the factor of a 4-bit one."""

    def __init__(self, ctx, rows: int, cols: int, experts: int, operands: str):
        self.ctx, self.operands, self.factor = ctx, operands, None
        if operands == "fp8":
            self.rows, self.cols = fp8.empty_rows(rows, cols), fp8.empty_cols(rows, cols, experts)
        else:
            self.rows, self.cols = fp4.empty_rows(rows, cols, format=operands, groups=experts), fp4.empty_cols(rows, cols, format=operands, groups=experts)
            if operands == "nvfp4":
                self.factor = torch.empty(1, device="cuda")

    def quantize(self, x, offsets, rows=None) -> None:
        if self.operands == "fp8":
            fp8.quantize_both(self.ctx, x, *self.rows, *self.cols, rows=rows, offsets=offsets)
            return
        if self.factor is not None:
            fp4.tensor_factor(self.ctx, x, self.factor)
        fp4.quantize_both(self.ctx, x, *self.rows, *self.cols, factor=self.factor, format=self.operands, rows=rows, offsets=offsets)


class _Weights:
    """A stack of weights as the products read it: ``rows`` for the forward, ``cols`` for the input gradient (8-bit tiles serve both)."""

    def __init__(self, ctx, w, operands: str):
        self.ctx, self.operands, self.factor = ctx, operands, None
        if operands == "fp8":
            self.rows = self.cols = fp8.empty_tiles(*w.shape)
        else:
            self.rows, self.cols = fp4.empty_rows(*w.shape, format=operands), fp4.empty_cols(*w.shape, format=operands)
            if operands == "nvfp4":
                self.factor = torch.empty(w.shape[0], device="cuda")
        self.half = None

    def __iter__(self):
        """The copy that the forward product reads, as a call takes it: ``plan.run(*x, *weights, y)``."""
        return iter(self.rows)

    def __getitem__(self, i):
        return self.rows[i]

    def __len__(self) -> int:
        return len(self.rows)

    def quantize(self, w) -> None:
        if self.operands == "fp8":
            fp8.quantize_tiles(self.ctx, w, *self.rows)
        else:
            if self.factor is not None:
                fp4.tensor_factor(self.ctx, w, self.factor)
            fp4.quantize_both(self.ctx, w, *self.rows, *self.cols, factor=self.factor, format=self.operands)
        if self.half is not None:
            self.half.copy_(w)

    def few(self, w):
        """As ``few_tokens`` takes them: the 4-bit row copies, or a half-precision copy that is made when it is first asked for."""
        if self.operands == "fp8":
            if self.half is None:
                self.half = w.half()
            return self.half
        return (*self.rows, self.factor)


class ExpertLayer:
    """y[t] = sum over the chosen experts e of w[t,e] * silu(x[t] W1[e]^T) W2[e]^T, with buffers and plans for one number of tokens (``close``
    gives the plans back).  operands: "fp8", "nvfp4" or "mxfp4"."""

    def __init__(self, ctx, tokens: int, hidden: int, inner: int, experts: int, top_k: int, seed: int = 0, operands: str = "fp8"):
        if operands not in OPERANDS:
            raise ValueError(f"operands must be one of {', '.join(OPERANDS)}")
        self.operands = operands
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.ctx, self.T, self.E, self.k = ctx, tokens, experts, top_k
        T, H, I, E, R = tokens, hidden, inner, experts, tokens * top_k
        new = lambda *s, dtype=torch.float32: torch.empty(*s, dtype=dtype, device="cuda")  # noqa: E731
        self.wr = (torch.randn(E, H, generator=g, device="cuda") * H ** -0.5).half()
        self.w1 = torch.randn(E, I, H, generator=g, device="cuda") * H ** -0.5
        self.w2 = torch.randn(E, H, I, generator=g, device="cuda") * I ** -0.5
        self.q1, self.q2 = _Weights(ctx, self.w1, operands), _Weights(ctx, self.w2, operands)
        self.refresh_weights()
        self.router_plan = ctx.plan(T, E, H)
        self.router = routing.Router(ctx, E, top_k, score="softmax", renormalize=True)
        self.logits, self.weights, self.indices = new(T, E, dtype=torch.float16), new(T, top_k), new(T, top_k, dtype=torch.int32)
        self.offsets, self.order, self.position = (new(n, dtype=torch.int32) for n in (E + 1, R, R))
        bf16 = torch.bfloat16
        if operands == "fp8":
            plan = lambda n, k, form, out: fp8.Plan(ctx, R, n, k, form=form, groups=E, out_dtype=out)  # noqa: E731
        else:
            plan = lambda n, k, form, out: fp4.Plan(ctx, R, n, k, form=form, groups=E, format=operands, out_dtype=out)  # noqa: E731
        self.up, self.down = plan(I, H, "forward", bf16), plan(H, I, "forward", bf16)
        self.up_dx, self.down_dx = plan(I, H, "input_grad", bf16), plan(H, I, "input_grad", bf16)
        self.up_dw, self.down_dw = plan(I, H, "weight_grad", torch.float32), plan(H, I, "weight_grad", torch.float32)
        self.h, self.y_rows = new(R, I, dtype=bf16), new(R, H, dtype=bf16)
        self.da, self.dx_rows = new(R, I, dtype=bf16), new(R, H, dtype=bf16)
        self.dw1, self.dw2, self.dlogits = new(E, I, H), new(E, H, I), new(T, E, dtype=torch.float16)
        self.xq, self.aq, self.dyq, self.dhq = (_Copies(ctx, R, n, E, operands) for n in (H, I, H, I))
        if operands == "fp8":                                                     # the 8-bit copies by names of their own: by rows and, per expert, by columns
            self.x8, self.a8, self.dy8, self.dh8 = (c.rows for c in (self.xq, self.aq, self.dyq, self.dhq))
            self.x8c, self.a8c, self.dy8c, self.dh8c = (c.cols for c in (self.xq, self.aq, self.dyq, self.dhq))
        self.few = few_tokens.Layer(ctx, H, I, E, top_k, weights="f16" if operands == "fp8" else operands, activation="silu", dtype=torch.float16)
        self.decode_plans, self.scratch = {}, None                                # made by the first decoding step

    def close(self) -> None:
        """Gives the plans back to the context."""
        for plan in (self.router_plan, self.up, self.down, self.up_dx, self.down_dx, self.up_dw, self.down_dw, *self.decode_plans.values()):
            plan.close()

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def refresh_weights(self) -> None:
        """After a change of the weights: their copies."""
        self.q1.quantize(self.w1)
        self.q2.quantize(self.w2)

    def _product(self, plan, a, b, out) -> None:
        """One product over the experts; a and b are (copy, factor)."""
        factors = {} if self.operands == "fp8" else {"a_factor": a[1], "b_factor": b[1]}
        plan.run(*a[0], *b[0], out, offsets=self.offsets, **factors)

    def forward(self, x):
        """x (tokens, hidden) fp16 -> y (tokens, hidden) fp32; keeps what the backward pass needs."""
        self.x = x
        self.router_plan.run(x, self.wr, self.logits)
        self.router.forward(self.logits, self.weights, self.indices)
        self.router.sort(self.indices, self.offsets, self.order, self.position)
        self.rows = torch.div(self.order, self.k, rounding_mode="floor").int()        # the token at each place of the expert order
        self.xq.quantize(x, self.offsets, rows=self.rows)
        self._product(self.up, (self.xq.rows, self.xq.factor), (self.q1.rows, self.q1.factor), self.h)
        self.a = torch.nn.functional.silu(self.h.float())
        self.aq.quantize(self.a, self.offsets)
        self._product(self.down, (self.aq.rows, self.aq.factor), (self.q2.rows, self.q2.factor), self.y_rows)
        picked = self.y_rows[self.position.long()].view(self.T, self.k, -1).float()
        return (self.weights.unsqueeze(-1) * picked).sum(1)

    def backward(self, dy):
        """dy (tokens, hidden) fp32 -> (dx, dw1, dw2, dlogits)."""
        place = self.position.long()
        dweights = (dy.unsqueeze(1) * self.y_rows[place].view(self.T, self.k, -1).float()).sum(-1)
        dy_rows = dy[self.rows.long()] * self.weights.flatten()[self.order.long()].unsqueeze(-1)
        self.dyq.quantize(dy_rows, self.offsets)
        self._product(self.down_dx, (self.dyq.rows, self.dyq.factor), (self.q2.cols, self.q2.factor), self.da)
        self._product(self.down_dw, (self.dyq.cols, self.dyq.factor), (self.aq.cols, self.aq.factor), self.dw2)
        h = self.h.float()
        s = torch.sigmoid(h)
        dh = self.da.float() * s * (1 + h * (1 - s))
        self.dhq.quantize(dh, self.offsets)
        self._product(self.up_dx, (self.dhq.rows, self.dhq.factor), (self.q1.cols, self.q1.factor), self.dx_rows)
        self._product(self.up_dw, (self.dhq.cols, self.dhq.factor), (self.xq.cols, self.xq.factor), self.dw1)
        self.router.backward(self.logits, self.indices, dweights, self.dlogits)
        dx = self.dx_rows[place].view(self.T, self.k, -1).float().sum(1) + self.dlogits.float() @ self.wr.float()
        return dx, self.dw1, self.dw2, self.dlogits

    def decode(self, x):
        """x (t, hidden) fp16, at most 64 tokens -> y (t, hidden) fp16; the training step's buffers stay as they are.  The first step of a number of tokens
        makes its plan, so it runs before one is captured into a graph; steps of one layer share scratch memory and run one after the other."""
        t = x.shape[0]
        if t > few_tokens.MAX_TOKENS:
            raise ValueError(f"at most {few_tokens.MAX_TOKENS} tokens, not {t}")
        y = torch.empty(t, self.few.hidden, dtype=torch.float16, device="cuda")
        if t == 0:
            return y
        if t not in self.decode_plans:
            self.decode_plans[t] = self.ctx.plan(t, self.E, self.few.hidden)
        if self.scratch is None:
            self.scratch = self.few.empty_scratch()
        logits = torch.empty(t, self.E, dtype=torch.float16, device="cuda")
        weights, indices = torch.empty(t, self.k, device="cuda"), torch.empty(t, self.k, dtype=torch.int32, device="cuda")
        self.decode_plans[t].run(x, self.wr, logits)
        self.router.forward(logits, weights, indices)
        self.few.run(x, self.q1.few(self.w1), self.q2.few(self.w2), indices, weights, y, self.scratch)
        return y


def main() -> None:
    ap = argparse.ArgumentParser()
    for name, value in (("tokens", 4096), ("hidden", 2048), ("inner", 1024), ("experts", 32), ("top-k", 4), ("iters", 5)):
        ap.add_argument(f"--{name}", type=int, default=value)
    ap.add_argument("--operands", choices=OPERANDS, default="fp8")
    ap.add_argument("--decode", type=int, default=0, help="also time a decoding step of so many tokens, 64 at most")
    args = ap.parse_args()
    with hgemm.Context(0) as ctx, ExpertLayer(ctx, args.tokens, args.hidden, args.inner, args.experts, args.top_k,
                                                operands=args.operands) as layer:
        x = torch.randn(args.tokens, args.hidden, device="cuda").half()
        dy = torch.randn(args.tokens, args.hidden, device="cuda")
        for _ in range(2):
            layer.forward(x)
            layer.backward(dy)
        e = [torch.cuda.Event(enable_timing=True) for _ in range(3)]
        times = []
        for _ in range(args.iters):
            e[0].record()
            layer.forward(x)
            e[1].record()
            layer.backward(dy)
            e[2].record()
            torch.cuda.synchronize()
            times.append((e[0].elapsed_time(e[1]) * 1e3, e[1].elapsed_time(e[2]) * 1e3))
        decode = ""
        if args.decode:
            graph = torch.cuda.CUDAGraph()                                        # a decoding step is launched from a graph
            few = x[:1].expand(args.decode, -1).contiguous() + torch.randn(args.decode, args.hidden, device="cuda").half()
            layer.decode(few)
            torch.cuda.synchronize()
            with torch.cuda.graph(graph):
                layer.decode(few)
            graph.replay()
            e[0].record()
            for _ in range(args.iters):
                graph.replay()
            e[1].record()
            torch.cuda.synchronize()
            decode = f", decoding {args.decode} tokens {e[0].elapsed_time(e[1]) * 1e3 / args.iters:.0f} us"
        status = ctx.last_device_status()
        f, b = sorted(t[0] for t in times)[len(times) // 2], sorted(t[1] for t in times)[len(times) // 2]
        print(f"{args.tokens} tokens, top {args.top_k} of {args.experts} experts, {args.hidden} -> {args.inner} -> {args.hidden}: "
              f"{args.operands} forward {f:.0f} us, backward {b:.0f} us{decode}, status {status}")


if __name__ == "__main__":
    main()

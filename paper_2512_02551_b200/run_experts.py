"""One training step of a layer of experts on the 8-bit products, end to end, and its device time.

    python -m paper_2512_02551_b200.run_experts [--tokens 4096] [--hidden 2048] [--inner 1024] [--experts 32] [--top-k 4] [--iters 5]

``ExpertLayer`` shows how the pieces fit: the router's logits are a half-precision product (``hgemm``), the routing chooses
and orders (``routing``), tokens are gathered into expert order and quantised in one pass (``fp8.quantize_*``), each expert's two
products run as one grouped launch (``fp8.Plan`` with groups), and the backward pass uses the same weights' tiles for the
input gradients and column copies laid out per expert for the weight gradients.
"""
from __future__ import annotations

import argparse

import torch

from . import fp8, hgemm, routing


class ExpertLayer:
    """y[t] = sum over the chosen experts e of w[t,e] * silu(x[t] W1[e]^T) W2[e]^T, with buffers and plans for one number of tokens (``close``
    gives the plans back)."""

    def __init__(self, ctx, tokens: int, hidden: int, inner: int, experts: int, top_k: int, seed: int = 0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.ctx, self.T, self.E, self.k = ctx, tokens, experts, top_k
        T, H, I, E, R = tokens, hidden, inner, experts, tokens * top_k
        new = lambda *s, dtype=torch.float32: torch.empty(*s, dtype=dtype, device="cuda")  # noqa: E731
        self.wr = (torch.randn(E, H, generator=g, device="cuda") * H ** -0.5).half()
        self.w1 = torch.randn(E, I, H, generator=g, device="cuda") * H ** -0.5
        self.w2 = torch.randn(E, H, I, generator=g, device="cuda") * I ** -0.5
        self.q1, self.q2 = fp8.empty_tiles(E, I, H), fp8.empty_tiles(E, H, I)
        self.refresh_weights()
        self.router_plan = ctx.plan(T, E, H)
        self.router = routing.Router(ctx, E, top_k, score="softmax", renormalize=True)
        self.logits, self.weights, self.indices = new(T, E, dtype=torch.float16), new(T, top_k), new(T, top_k, dtype=torch.int32)
        self.offsets, self.order, self.position = (new(n, dtype=torch.int32) for n in (E + 1, R, R))
        bf16 = torch.bfloat16
        plan = lambda n, k, form, out: fp8.Plan(ctx, R, n, k, form=form, groups=E, out_dtype=out)  # noqa: E731
        self.up, self.down = plan(I, H, "forward", bf16), plan(H, I, "forward", bf16)
        self.up_dx, self.down_dx = plan(I, H, "input_grad", bf16), plan(H, I, "input_grad", bf16)
        self.up_dw, self.down_dw = plan(I, H, "weight_grad", torch.float32), plan(H, I, "weight_grad", torch.float32)
        self.h, self.y_rows = new(R, I, dtype=bf16), new(R, H, dtype=bf16)
        self.da, self.dx_rows = new(R, I, dtype=bf16), new(R, H, dtype=bf16)
        self.dw1, self.dw2, self.dlogits = new(E, I, H), new(E, H, I), new(T, E, dtype=torch.float16)
        # 8-bit copies by rows and, per expert, by columns
        self.x8, self.a8, self.dy8, self.dh8 = (fp8.empty_rows(R, n) for n in (H, I, H, I))
        self.x8c, self.a8c, self.dy8c, self.dh8c = (fp8.empty_cols(R, n, E) for n in (H, I, H, I))

    def close(self) -> None:
        """Gives the plans back to the context."""
        for plan in (self.router_plan, self.up, self.down, self.up_dx, self.down_dx, self.up_dw, self.down_dw):
            plan.close()

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def refresh_weights(self) -> None:
        """After a change of the weights: their 8-bit tiles."""
        fp8.quantize_tiles(self.ctx, self.w1, *self.q1)
        fp8.quantize_tiles(self.ctx, self.w2, *self.q2)

    def forward(self, x):
        """x (tokens, hidden) fp16 -> y (tokens, hidden) fp32; keeps what the backward pass needs."""
        ctx = self.ctx
        self.x = x
        self.router_plan.run(x, self.wr, self.logits)
        self.router.forward(self.logits, self.weights, self.indices)
        self.router.sort(self.indices, self.offsets, self.order, self.position)
        self.rows = torch.div(self.order, self.k, rounding_mode="floor").int()        # the token at each place of the expert order
        fp8.quantize_both(ctx, x, *self.x8, *self.x8c, rows=self.rows, offsets=self.offsets)
        self.up.run(*self.x8, *self.q1, self.h, offsets=self.offsets)
        self.a = torch.nn.functional.silu(self.h.float())
        fp8.quantize_both(ctx, self.a, *self.a8, *self.a8c, offsets=self.offsets)
        self.down.run(*self.a8, *self.q2, self.y_rows, offsets=self.offsets)
        picked = self.y_rows[self.position.long()].view(self.T, self.k, -1).float()
        return (self.weights.unsqueeze(-1) * picked).sum(1)

    def backward(self, dy):
        """dy (tokens, hidden) fp32 -> (dx, dw1, dw2, dlogits)."""
        ctx, place = self.ctx, self.position.long()
        dweights = (dy.unsqueeze(1) * self.y_rows[place].view(self.T, self.k, -1).float()).sum(-1)
        dy_rows = dy[self.rows.long()] * self.weights.flatten()[self.order.long()].unsqueeze(-1)
        fp8.quantize_both(ctx, dy_rows, *self.dy8, *self.dy8c, offsets=self.offsets)
        self.down_dx.run(*self.dy8, *self.q2, self.da, offsets=self.offsets)
        self.down_dw.run(*self.dy8c, *self.a8c, self.dw2, offsets=self.offsets)
        h = self.h.float()
        s = torch.sigmoid(h)
        dh = self.da.float() * s * (1 + h * (1 - s))
        fp8.quantize_both(ctx, dh, *self.dh8, *self.dh8c, offsets=self.offsets)
        self.up_dx.run(*self.dh8, *self.q1, self.dx_rows, offsets=self.offsets)
        self.up_dw.run(*self.dh8c, *self.x8c, self.dw1, offsets=self.offsets)
        self.router.backward(self.logits, self.indices, dweights, self.dlogits)
        dx = self.dx_rows[place].view(self.T, self.k, -1).float().sum(1) + self.dlogits.float() @ self.wr.float()
        return dx, self.dw1, self.dw2, self.dlogits


def main() -> None:
    ap = argparse.ArgumentParser()
    for name, value in (("tokens", 4096), ("hidden", 2048), ("inner", 1024), ("experts", 32), ("top-k", 4), ("iters", 5)):
        ap.add_argument(f"--{name}", type=int, default=value)
    args = ap.parse_args()
    with hgemm.Context(0) as ctx, ExpertLayer(ctx, args.tokens, args.hidden, args.inner, args.experts, args.top_k) as layer:
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
        status = ctx.last_device_status()
        f, b = sorted(t[0] for t in times)[len(times) // 2], sorted(t[1] for t in times)[len(times) // 2]
        print(f"{args.tokens} tokens, top {args.top_k} of {args.experts} experts, {args.hidden} -> {args.inner} -> {args.hidden}: "
              f"forward {f:.0f} us, backward {b:.0f} us, status {status}")


if __name__ == "__main__":
    main()

"""A mixture-of-experts feed-forward layer, for serving and for training.

Serving (``ServingLayer``): expert weights in 4 bits.  The router's choices are
sorted by expert, the gate and up projections read the tokens' rows through the
sorted order and apply silu(gate) * up, the down projection follows on the
sorted rows, and the experts' rows are summed back into the tokens with the
router's weights: four calls, five launches at most.

Training (``TrainingLayer``): expert weights in bfloat16 and plain matrix
products over each expert's rows; rows go out and come back through
``dispatch`` and ``combine``, whose gradients are the library's too.

Run it on an MI355X:  python examples/moe_layer.py [--tokens 32] [--experts 64]
It prints how far the 4-bit layer is from one with the same weights in 32 bits,
whether gradients match a plain computation, and the time of a serving step.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch
from torch.autograd.function import once_differentiable

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))

import paper_2305_06942_amd as ebag  # noqa: E402


def route(logits, choices):
    """(expert of each choice int32, weight of each choice float32) [tokens, choices]."""
    top, experts = logits.topk(choices, dim=1)
    return experts.int().contiguous(), torch.softmax(top.float(), dim=1)


class Order:
    """The choices of up to max_tokens tokens in the order of their experts."""

    def __init__(self, max_tokens, choices, experts):
        self.plan = ebag.MoePerm(max_tokens, choices, experts)
        self.choices, self.experts = choices, experts

    def sort(self, expert_of):
        new = lambda *shape: torch.empty(shape, dtype=torch.int32, device=expert_of.device)  # noqa: E731
        offsets, pos, src = new(self.experts + 1), new(*expert_of.shape), new(expert_of.numel())
        self.plan.sort(expert_of, offsets, pos, src)
        return offsets, pos, src


class ServingLayer:
    """gate_up [experts, 2 * hidden, dim] (gate rows first) and down [experts,
    dim, hidden], rounded to 4 bits with a scale and zero for every `group` columns."""

    def __init__(self, gate_up, down, choices, max_tokens, group=128):
        experts, twice, dim = gate_up.shape
        self.dim, self.hidden = dim, twice // 2
        self.order = Order(max_tokens, choices, experts)
        kind = {torch.float32: ebag.EBAG_F32, torch.float16: ebag.EBAG_F16, torch.bfloat16: ebag.EBAG_BF16}[gate_up.dtype]
        self.up = ebag.Q4Gemv(twice, dim, group, kind, experts=experts, glu=1)
        self.down = ebag.Q4Gemv(dim, self.hidden, group, kind, experts=experts)
        self.up_weights = self._round(self.up, gate_up, group)
        self.down_weights = self._round(self.down, down, group)

    @staticmethod
    def _round(product, w, group):
        experts, rows, columns = w.shape
        groups = -(-columns // group)
        codes = torch.empty((experts, rows, (columns + 1) // 2), dtype=torch.uint8, device=w.device)
        scales = torch.empty((experts, rows, groups), dtype=w.dtype, device=w.device)
        zeros = torch.empty((experts, rows, groups), dtype=torch.uint8, device=w.device)
        product.quantize(w.contiguous(), codes, scales, zeros)
        return codes, scales, zeros

    def __call__(self, x, logits):
        choices = self.order.choices
        expert_of, weights = route(logits, choices)
        offsets, pos, src = self.order.sort(expert_of)
        h = torch.empty((src.numel(), self.hidden), dtype=x.dtype, device=x.device)
        ys = torch.empty((src.numel(), self.dim), dtype=x.dtype, device=x.device)
        out = torch.empty_like(x)
        self.up.experts(*self.up_weights, x, offsets, h, src=src, k=choices)
        self.down.experts(*self.down_weights, h, offsets, ys)
        self.order.plan.combine(ys, offsets, pos, weights, out)
        return out


class _Dispatch(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, plan, offsets, pos):
        xs = torch.empty((pos.numel(), x.shape[1]), dtype=x.dtype, device=x.device)
        plan.dispatch(x, offsets, pos, xs)
        ctx.plan, ctx.shape = plan, x.shape
        ctx.save_for_backward(offsets, pos)
        return xs

    @staticmethod
    @once_differentiable
    def backward(ctx, dxs):
        offsets, pos = ctx.saved_tensors
        dx = torch.empty(ctx.shape, dtype=dxs.dtype, device=dxs.device)
        ctx.plan.dispatch_backward(dxs.contiguous(), offsets, pos, dx)
        return dx, None, None, None


class _Combine(torch.autograd.Function):
    @staticmethod
    def forward(ctx, ys, weights, plan, offsets, pos):
        out = torch.empty((pos.shape[0], ys.shape[1]), dtype=ys.dtype, device=ys.device)
        plan.combine(ys, offsets, pos, weights, out)
        ctx.plan = plan
        ctx.save_for_backward(ys, weights, offsets, pos)
        return out

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        ys, weights, offsets, pos = ctx.saved_tensors
        dys, dweights = torch.empty_like(ys), torch.empty_like(weights)
        ctx.plan.combine_backward(dout.contiguous(), ys, offsets, pos, weights, dys, dweights)
        return dys, dweights, None, None, None


class TrainingLayer(torch.nn.Module):
    def __init__(self, gate_up, down, choices, max_tokens):
        super().__init__()
        self.gate_up, self.down = torch.nn.Parameter(gate_up.clone()), torch.nn.Parameter(down.clone())
        self.order = Order(max_tokens, choices, gate_up.shape[0])

    def forward(self, x, logits):
        expert_of, weights = route(logits, self.order.choices)
        offsets, pos, _ = self.order.sort(expert_of)
        xs = _Dispatch.apply(x, self.order.plan, offsets, pos)
        ends = offsets.tolist()
        parts = []
        for e in range(self.order.experts):
            gate, up = (xs[ends[e]:ends[e + 1]] @ self.gate_up[e].t()).chunk(2, dim=1)
            parts.append((torch.nn.functional.silu(gate) * up) @ self.down[e].t())
        return _Combine.apply(torch.cat(parts), weights, self.order.plan, offsets, pos)


def plain_layer(x, logits, gate_up, down, choices):
    """The layer in plain torch operations, token by token's choice, in x's type."""
    expert_of, weights = route(logits, choices)
    out = torch.zeros_like(x)
    for j in range(choices):
        gate, up = torch.bmm(gate_up[expert_of[:, j].long()], x[:, :, None])[..., 0].chunk(2, dim=1)
        y = torch.bmm(down[expert_of[:, j].long()], (torch.nn.functional.silu(gate) * up)[:, :, None])[..., 0]
        out = out + weights[:, j, None].to(x.dtype) * y
    return out


def rounded(product, weights):
    """The values that a product's 4-bit weights stand for, float32."""
    codes, scales, zeros = weights
    q = torch.stack((codes & 15, codes >> 4), -1).flatten(-2)[..., :product.K].float()
    column = torch.arange(product.K, device=codes.device) // product.group
    return scales.float()[..., column] * (q - zeros.float()[..., column])


def make(tokens, experts, choices, dim, hidden, seed=0, dtype=torch.bfloat16, device="cuda"):
    g = torch.Generator(device=device).manual_seed(seed)
    normal = lambda *shape: torch.randn(shape, generator=g, device=device)  # noqa: E731
    return ((normal(experts, 2 * hidden, dim) / dim ** 0.5).to(dtype), (normal(experts, dim, hidden) / hidden ** 0.5).to(dtype),
            normal(tokens, dim).to(dtype), normal(tokens, experts))


def serving_error(tokens, experts, choices, dim, hidden, **kw):
    """Relative distance of the 4-bit layer from the same weights' in 32 bits."""
    gate_up, down, x, logits = make(tokens, experts, choices, dim, hidden, **kw)
    layer = ServingLayer(gate_up, down, choices, tokens)
    got = layer(x, logits).float()
    want = plain_layer(x.float(), logits, rounded(layer.up, layer.up_weights),
                       rounded(layer.down, layer.down_weights), choices)
    return float((got - want).norm() / want.norm())


def gradient_errors(tokens, experts, choices, dim, hidden, **kw):
    """Relative distances of the training layer's output and gradients from a plain computation's."""
    gate_up, down, x, logits = make(tokens, experts, choices, dim, hidden, **kw)
    layer = TrainingLayer(gate_up, down, choices, tokens)
    x1, l1 = x.clone().requires_grad_(), logits.clone().requires_grad_()
    x2, l2 = x.clone().requires_grad_(), logits.clone().requires_grad_()
    g2, d2 = gate_up.clone().requires_grad_(), down.clone().requires_grad_()
    dout = torch.randn_like(x)
    out = layer(x1, l1)
    out.backward(dout)
    want = plain_layer(x2, l2, g2, d2, choices)
    want.backward(dout)
    far = lambda a, b: float((a - b).detach().float().norm() / b.detach().float().norm())  # noqa: E731
    return {"out": far(out, want), "x": far(x1.grad, x2.grad), "logits": far(l1.grad, l2.grad),
            "gate_up": far(layer.gate_up.grad, g2.grad), "down": far(layer.down.grad, d2.grad)}


def main():
    p = argparse.ArgumentParser()
    p.add_argument("--tokens", type=int, default=32)
    p.add_argument("--experts", type=int, default=64)
    p.add_argument("--choices", type=int, default=8)
    p.add_argument("--dim", type=int, default=2048)
    p.add_argument("--hidden", type=int, default=1024)
    a = p.parse_args()
    torch.cuda.set_device(0)
    print(f"4-bit layer against its weights in 32 bits: {serving_error(a.tokens, a.experts, a.choices, a.dim, a.hidden):.1e}")
    errors = gradient_errors(64, 8, 2, 256, 128, dtype=torch.float32)
    print("gradients against a plain computation: " + ", ".join(f"{n} {e:.1e}" for n, e in errors.items()))
    gate_up, down, x, logits = make(a.tokens, a.experts, a.choices, a.dim, a.hidden)
    layer = ServingLayer(gate_up, down, a.choices, a.tokens)
    for _ in range(10):
        layer(x, logits)
    begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    begin.record()
    for _ in range(100):
        layer(x, logits)
    end.record()
    torch.cuda.synchronize()
    print(f"a step of {a.tokens} tokens, {a.experts} experts of 3 x {a.dim} x {a.hidden}: {begin.elapsed_time(end) * 10:.1f} us")


if __name__ == "__main__":
    main()

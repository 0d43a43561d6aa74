"""A mixture-of-experts feed-forward layer, for serving and for training.

Serving (``ServingLayer``): expert weights in 4 bits, or in 8 with the rows
rounded to 8 bits too.  The router chooses each token's experts and weights, the
choices are sorted by expert, the gate and up projections read the tokens' rows
through the sorted order and apply silu(gate) * up, the down projection follows on
the sorted rows, and the experts' rows are summed back into the tokens with the
router's weights: five calls, six launches at most with 4 bits, eight with 8.

Training (``TrainingLayer``): expert weights in bfloat16 and plain matrix
products over each expert's rows; choices and weights come from ``choose``, which
also makes the balance loss and the loss that keeps logits small, rows go out and
come back through ``dispatch`` and ``combine``, and all gradients are the library's.

Run it on an MI355X:  python examples/moe_layer.py [--tokens 32] [--experts 64]
It prints how far the layers in 4 and 8 bits are from one with the same weights in
32 bits, whether gradients match a plain computation, and the time of a serving step.
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
    """(expert of each choice int32, weight of each choice float32) [tokens, choices], in plain torch operations."""
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

    @staticmethod
    def readable(logits):
        """Logits as the library's router takes them: of other types as float32, and with rows of adjacent columns that do not
        overlap."""
        if logits.dtype not in (torch.float32, torch.float16, torch.bfloat16):
            logits = logits.float()
        return logits if logits.stride(1) == 1 and logits.stride(0) >= logits.shape[1] else logits.contiguous()

    def choose(self, logits):
        """(experts int32, weights float32) [tokens, choices]; a token's weights add up to 1."""
        logits = self.readable(logits)
        shape = (logits.shape[0], self.choices)
        ids = torch.empty(shape, dtype=torch.int32, device=logits.device)
        weights = torch.empty(shape, dtype=torch.float32, device=logits.device)
        self.plan.choose(logits, ids, weights)
        return ids, weights


class ServingLayer:
    """gate_up [experts, 2 * hidden, dim] (gate rows first) and down [experts,
    dim, hidden], rounded to 4 bits with a scale and zero for every `group` columns,
    or to 8 with a scale for every row."""

    def __init__(self, gate_up, down, choices, max_tokens, group=128, bits=4):
        experts, twice, dim = gate_up.shape
        self.dim, self.hidden, self.bits = dim, twice // 2, bits
        self.order = Order(max_tokens, choices, experts)
        kind = {torch.float32: ebag.EBAG_F32, torch.float16: ebag.EBAG_F16, torch.bfloat16: ebag.EBAG_BF16}[gate_up.dtype]
        if bits == 8:
            self.up = ebag.Q8Gemv(twice, dim, kind, experts=experts, glu=1)
            self.down = ebag.Q8Gemv(dim, self.hidden, kind, experts=experts)
            self.up_weights, self.down_weights = self._round8(self.up, gate_up), self._round8(self.down, down)
            return
        self.up = ebag.Q4Gemv(twice, dim, group, kind, experts=experts, glu=1)
        self.down = ebag.Q4Gemv(dim, self.hidden, group, kind, experts=experts)
        self.up_weights = self._round(self.up, gate_up, group)
        self.down_weights = self._round(self.down, down, group)

    @staticmethod
    def _round8(product, w):
        codes = torch.empty((*w.shape[:2], product.pitch), dtype=torch.int8, device=w.device)
        scales = torch.empty(w.shape[:2], dtype=torch.float32, device=w.device)
        product.quantize(w.contiguous(), codes, scales)
        return codes, scales

    def _multiply(self, product, weights, x, offsets, y, src=None):
        k = self.order.choices if src is not None else 1
        if self.bits == 4:
            product.experts(*weights, x, offsets, y, src=src, k=k)
            return
        xq = torch.empty((x.shape[0], product.pitch), dtype=torch.int8, device=x.device)
        xs = torch.empty(x.shape[0], dtype=torch.float32, device=x.device)
        product.experts(*weights, x, offsets, y, xq, xs, src=src, k=k)

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
        expert_of, weights = self.order.choose(logits)
        offsets, pos, src = self.order.sort(expert_of)
        h = torch.empty((src.numel(), self.hidden), dtype=x.dtype, device=x.device)
        ys = torch.empty((src.numel(), self.dim), dtype=x.dtype, device=x.device)
        out = torch.empty_like(x)
        self._multiply(self.up, self.up_weights, x, offsets, h, src)
        self._multiply(self.down, self.down_weights, h, offsets, ys)
        self.order.plan.combine(ys, offsets, pos, weights, out)
        return out


class _Choose(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, plan, live):
        new = lambda *shape, dtype=torch.float32: torch.empty(shape, dtype=dtype, device=logits.device)  # noqa: E731
        n, k, experts = logits.shape[0], plan.choices, plan.experts
        ids, counts = new(n, k, dtype=torch.int32), new(experts + 1, dtype=torch.int32)
        weights, losses = new(n, k), new(2)
        plan.choose(logits, ids, weights, counts, new(experts + 1), losses, new(plan.choose_work), live=live)
        ctx.plan = plan
        ctx.save_for_backward(logits, ids, counts, live)
        ctx.mark_non_differentiable(ids)
        return ids, weights, losses

    @staticmethod
    @once_differentiable
    def backward(ctx, _, dweights, dlosses):
        logits, ids, counts, live = ctx.saved_tensors
        dlogits = torch.empty_like(logits)
        ctx.plan.choose_backward(logits, ids, dweights.contiguous(), dlogits, counts=counts, dlosses=dlosses.contiguous(), live=live)
        return dlogits, None, None


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

    def forward(self, x, logits, live=None):
        return self.with_losses(x, logits, live)[0]

    def with_losses(self, x, logits, live=None):
        """(the layer's output, float32 [2]: the balance loss and the mean square of the logits' log-sum).  live: which
        tokens of a padded batch count; the others' rows of the output are zeros."""
        expert_of, weights, losses = _Choose.apply(self.order.readable(logits).contiguous(), self.order.plan, live)
        offsets, pos, _ = self.order.sort(expert_of)
        xs = _Dispatch.apply(x, self.order.plan, offsets, pos)
        ends = offsets.tolist()
        parts = []
        for e in range(self.order.experts):
            gate, up = (xs[ends[e]:ends[e + 1]] @ self.gate_up[e].t()).chunk(2, dim=1)
            parts.append((torch.nn.functional.silu(gate) * up) @ self.down[e].t())
        parts.append(xs[ends[-1]:].new_zeros(xs.shape[0] - ends[-1], self.down.shape[1]))  # of choices that no expert takes
        return _Combine.apply(torch.cat(parts), weights, self.order.plan, offsets, pos), losses


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


def plain_losses(logits, choices, live=None):
    """Both losses of the router in plain torch operations."""
    if live is not None:
        logits = logits[live]
    p, counts = torch.softmax(logits.float(), dim=1), torch.zeros_like(logits[0], dtype=torch.float32)
    ids = logits.topk(choices, dim=1).indices.reshape(-1)
    counts = counts.index_add(0, ids, torch.ones_like(ids, dtype=torch.float32))
    n, experts = logits.shape
    return torch.stack((experts / (choices * n * n) * (counts * p.sum(0)).sum(), torch.logsumexp(logits.float(), dim=1).square().mean()))


def eight_bits(x):
    """The values that rows rounded to 8 bits stand for, float32."""
    scale = (x.double().abs().amax(-1, keepdim=True) / 127).float()
    return torch.round(x.double() / torch.where(scale > 0, scale, 1.0).double()).clamp(-127, 127).float() * scale


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


def serving_error_8(tokens, experts, choices, dim, hidden, **kw):
    """The same for the 8-bit layer, with the reference's rows rounded to 8 bits where the layer's are."""
    gate_up, down, x, logits = make(tokens, experts, choices, dim, hidden, **kw)
    layer = ServingLayer(gate_up, down, choices, tokens, bits=8)
    got = layer(x, logits).float()
    expert_of, weights = route(logits, choices)
    want = torch.zeros_like(got)
    values = lambda product, w: w[0][..., :product.K].float() * w[1][..., None]  # noqa: E731
    up, down8 = values(layer.up, layer.up_weights), values(layer.down, layer.down_weights)
    for j in range(choices):
        e = expert_of[:, j].long()
        gate, ups = torch.bmm(up[e], eight_bits(x)[:, :, None])[..., 0].chunk(2, dim=1)
        y = torch.bmm(down8[e], eight_bits(torch.nn.functional.silu(gate) * ups)[:, :, None])[..., 0]
        want = want + weights[:, j, None] * y
    return float((got - want).norm() / want.norm())


def loss_gradient_error(tokens, experts, choices, dim, hidden, padded=0.0, **kw):
    """Relative distances of the losses, and of the logits' gradient of output and losses together, from a plain computation's."""
    gate_up, down, x, logits = make(tokens, experts, choices, dim, hidden, **kw)
    live = torch.rand(tokens, generator=torch.Generator(device=x.device).manual_seed(3), device=x.device) >= padded if padded else None
    layer = TrainingLayer(gate_up, down, choices, tokens)
    l1, l2 = logits.clone().requires_grad_(), logits.clone().requires_grad_()
    dout = torch.randn_like(x)
    coefficients = torch.tensor((0.5, 0.25), device=x.device)
    out, losses = layer.with_losses(x, l1, live)
    ((out * dout).sum() / tokens + (losses * coefficients).sum()).backward()
    want = plain_losses(l2, choices, live)
    keep = 1.0 if live is None else live[:, None].float()
    ((plain_layer(x, l2, gate_up, down, choices) * dout * keep).sum() / tokens + (want * coefficients).sum()).backward()
    far = lambda a, b: float((a - b).detach().float().norm() / b.detach().float().norm())  # noqa: E731
    return {"losses": far(losses, want), "logits": far(l1.grad, l2.grad)}


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
    print(f"8-bit layer against its weights and rows in 32 bits: {serving_error_8(a.tokens, a.experts, a.choices, a.dim, a.hidden):.1e}")
    errors = gradient_errors(64, 8, 2, 256, 128, dtype=torch.float32)
    print("gradients against a plain computation: " + ", ".join(f"{n} {e:.1e}" for n, e in errors.items()))
    errors = loss_gradient_error(64, 8, 2, 256, 128, padded=0.2, dtype=torch.float32)
    print("with the router's losses: " + ", ".join(f"{n} {e:.1e}" for n, e in errors.items()))
    gate_up, down, x, logits = make(a.tokens, a.experts, a.choices, a.dim, a.hidden)
    for bits in (4, 8):
        layer = ServingLayer(gate_up, down, a.choices, a.tokens, bits=bits)
        for _ in range(10):
            layer(x, logits)
        begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        begin.record()
        for _ in range(100):
            layer(x, logits)
        end.record()
        torch.cuda.synchronize()
        print(f"a step of {a.tokens} tokens, {a.experts} experts of 3 x {a.dim} x {a.hidden} in {bits} bits: "
              f"{begin.elapsed_time(end) * 10:.1f} us")


if __name__ == "__main__":
    main()

"""The example's layers take logits of any floating type and layout."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    import importlib.util
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    torch.cuda.set_device(0)
    spec = importlib.util.spec_from_file_location("moe_layer_logits", os.path.join(ROOT, "examples", "moe_layer.py"))
    module = importlib.util.module_from_spec(spec)
    sys.modules["moe_layer_logits"] = module
    spec.loader.exec_module(module)
    yield module
    torch.cuda.synchronize()


def _layouts(logits):
    """The same numbers as fp64, with columns that are not adjacent, with rows apart, and with columns in steps."""
    wide = logits.new_zeros((logits.shape[0], 3 * logits.shape[1]))
    wide[:, ::3] = logits
    apart = logits.new_zeros((logits.shape[0], logits.shape[1] + 3))
    apart[:, 1:-2] = logits
    return {"fp64": logits.double(), "transposed": logits.t().contiguous().t(), "steps": wide[:, ::3], "apart": apart[:, 1:-2],
            "fp64 transposed": logits.double().t().contiguous().t()}


@pytest.mark.parametrize("bits", [4, 8])
def test_serving(example, bits):
    import torch
    gate_up, down, x, logits = example.make(37, 6, 2, 64, 32)
    layer = example.ServingLayer(gate_up, down, 2, 37, bits=bits)
    want = layer(x, logits)
    for name, l in _layouts(logits).items():
        assert torch.equal(layer(x, l), want), name
    one = logits[:1].expand(37, -1)  # rows in the same memory
    assert torch.equal(layer(x, one), layer(x, one.contiguous()))


def test_training(example):
    import torch
    gate_up, down, x, logits = example.make(37, 6, 2, 64, 32, dtype=torch.float32)
    layer = example.TrainingLayer(gate_up, down, 2, 37)
    dout = torch.randn_like(x)

    def gradient(l):
        leaf = l.detach().requires_grad_()
        out, losses = layer.with_losses(x, leaf)
        ((out * dout).sum() + losses.sum()).backward()
        assert leaf.grad.dtype == l.dtype
        return out.detach(), losses.detach(), leaf.grad.float()

    want = gradient(logits)
    for name, l in _layouts(logits).items():
        assert all(torch.equal(a, b) for a, b in zip(gradient(l), want)), name
    leaf = logits[:1].detach().requires_grad_()
    layer(x, leaf.expand(37, -1)).sum().backward()
    assert leaf.grad.isfinite().all()


@pytest.mark.parametrize("what", ["live", "logits"])
def test_what_the_gradient_needs_is_not_changed_in_between(example, what):
    """autograd refuses the backward pass of a call whose mask or logits were written to since."""
    import torch
    gate_up, down, x, logits = example.make(20, 6, 2, 64, 32, dtype=torch.float32)
    layer = example.TrainingLayer(gate_up, down, 2, 20)
    leaf = logits.requires_grad_()
    live = torch.arange(20, device="cuda") % 3 > 0
    out, losses = layer.with_losses(x, leaf, live)
    (out.sum() + losses.sum()).backward(retain_graph=True)
    with torch.no_grad():
        {"live": live, "logits": leaf}[what].zero_()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        (out.sum() + losses.sum()).backward()

"""The example's layer with the library's router, its losses, and 8-bit weights.

8 bits: the reference rounds the same rows to 8 bits, but of the hidden rows it
rounds the values themselves and the layer their bfloat16 roundings, up to 2^-9 |h|
off.  Such a difference moves a code, by one step s = max|h| / 127, with a probability of 2^-9
|h| / s: a mean square of 2^-9 mean|h| s.  With max|h| up to 16 times and mean|h| up to the root
mean square that is 2^-9 * 16 / 127 = 2.5e-4 of the hidden rows' square, 1.6e-2 of their norm, and the
product carries it on; three roundings to bfloat16 add 2^-8: below 2^-5 together.

Losses and gradients in fp32: as in test_gpu_moe_layer.py, 1024 * 2^-24 of the norm."""
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
    spec = importlib.util.spec_from_file_location("moe_layer_router", os.path.join(ROOT, "examples", "moe_layer.py"))
    module = importlib.util.module_from_spec(spec)
    sys.modules["moe_layer_router"] = module
    spec.loader.exec_module(module)
    yield module
    torch.cuda.synchronize()


@pytest.mark.parametrize("tokens,experts,choices,dim,hidden", [
    (1, 8, 2, 256, 128), (32, 16, 4, 500, 130), (300, 5, 2, 512, 384), (700, 4, 2, 256, 640)])
def test_serving_layer_in_8_bits(example, tokens, experts, choices, dim, hidden):
    assert example.serving_error_8(tokens, experts, choices, dim, hidden) < 2.0 ** -5


@pytest.mark.parametrize("padded", [0.0, 0.3])
@pytest.mark.parametrize("tokens,experts,choices,dim,hidden", [(64, 8, 2, 256, 128), (50, 40, 6, 100, 60)])
def test_losses_and_their_gradient(example, tokens, experts, choices, dim, hidden, padded):
    import torch
    for name, e in example.loss_gradient_error(tokens, experts, choices, dim, hidden, padded=padded, dtype=torch.float32).items():
        assert e < 1024 * 2.0 ** -24, f"{name}: {e}"


def test_second_derivatives_raise(example):
    import torch
    gate_up, down, x, logits = example.make(8, 4, 2, 32, 16, dtype=torch.float32)
    layer = example.TrainingLayer(gate_up, down, 2, 8)
    leaf = logits.clone().requires_grad_()
    _, losses = layer.with_losses(x, leaf)
    first, = torch.autograd.grad(losses.sum(), leaf, create_graph=True)
    with pytest.raises(RuntimeError):
        torch.autograd.grad(first.sum(), leaf)

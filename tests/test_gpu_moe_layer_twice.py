"""The example's training layer differentiated twice: its gradients' kernels
are no autograd operations, so a second derivative through them must be
refused, not given without their part."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("of", ["gate_up", "down"])
def test_second_derivatives_are_refused(of):
    import torch
    torch.cuda.set_device(0)
    spec = importlib.util.spec_from_file_location("moe_layer_twice", os.path.join(ROOT, "examples", "moe_layer.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    gate_up, down, x, logits = example.make(12, 4, 2, 64, 32, dtype=torch.float32)
    layer = example.TrainingLayer(gate_up, down, 2, 12)
    x.requires_grad_()
    inputs = {"gate_up": layer.gate_up, "down": layer.down}
    loss = layer(x, logits).square().sum()
    first, = torch.autograd.grad(loss, inputs[of], create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        first.square().sum().backward()

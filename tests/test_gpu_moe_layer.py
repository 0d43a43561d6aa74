"""The example's mixture-of-experts layer: every operator in the place it has
in a model.

Serving: the two products and the sum round to bfloat16 once each (2^-8 at most,
a third of that as a root mean square), the reference not at all: three such
roundings stay below 2^-7 of the result's norm.  Training in fp32: sums of up
to 512 terms in another order, twice one after the other, stay below 1024 *
2^-24 of the norm, and silu's exponential adds a few units in the last place."""
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
    spec = importlib.util.spec_from_file_location("moe_layer", os.path.join(ROOT, "examples", "moe_layer.py"))
    module = importlib.util.module_from_spec(spec)
    sys.modules["moe_layer"] = module
    spec.loader.exec_module(module)
    yield module
    torch.cuda.synchronize()


@pytest.mark.parametrize("tokens,experts,choices,dim,hidden", [
    (1, 8, 2, 256, 128), (32, 16, 4, 500, 130), (300, 5, 2, 512, 384)])
def test_serving_layer(example, tokens, experts, choices, dim, hidden):
    assert example.serving_error(tokens, experts, choices, dim, hidden) < 2.0 ** -7


@pytest.mark.parametrize("tokens,experts,choices,dim,hidden", [(64, 8, 2, 256, 128), (5, 40, 6, 100, 60)])
def test_training_layer(example, tokens, experts, choices, dim, hidden):
    import torch
    for name, e in example.gradient_errors(tokens, experts, choices, dim, hidden, dtype=torch.float32).items():
        assert e < 1024 * 2.0 ** -24, f"{name}: {e}"

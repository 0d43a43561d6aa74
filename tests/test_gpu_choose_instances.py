"""Every instance of the router's kernels for many tokens, forward (with and without totals) and gradient, with the checks and
bounds of test_gpu_choose.py: 4 to 32 lanes of 16 logits a token, for one and two choices or more than 16, three to eight, and
nine to 16; workgroups of 256, 512 and 1024 threads; one turn and several."""
import pytest

from tests.test_gpu_choose import test_choose_and_gradient as whole_check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    torch.cuda.set_device(0)
    yield
    torch.cuda.synchronize()


CASES = [  # tokens, choices, experts, type, step, shift, masked, padded, bias, few
    (33000, 2, 60, "bfloat16", 0, 0, 0.3, 0.2, True, 0), (33000, 30, 60, "float32", 0, 0, 0, 0, False, 0), (33000, 50, 60, "float16", 0, 0, 0.5, 0, False, 7),
    (34000, 5, 50, "float32", 1, 1, 0, 0.1, True, 0), (33000, 12, 60, "float16", 0, 0, 0.6, 0, False, 9),
    (17000, 1, 65, "float16", 3, 0, 0, 0, True, 0), (17000, 2, 100, "float32", 0, 0, 0, 0.2, False, 5), (17000, 33, 120, "bfloat16", 0, 0, 0.5, 0, True, 0),
    (17000, 8, 128, "float32", 0, 0, 0, 0, False, 0), (17000, 8, 128, "bfloat16", 0, 0, 0.4, 0.3, True, 6), (17000, 3, 127, "float16", 1, 1, 0.98, 0, False, 0),
    (17000, 16, 70, "float32", 2, 0, 0, 0, True, 0), (8200, 1, 256, "bfloat16", 0, 0, 0, 0, False, 4), (8200, 7, 129, "float16", 5, 3, 0, 0.1, True, 0),
    (8200, 10, 200, "float32", 0, 0, 0.3, 0, True, 0), (5000, 2, 400, "float32", 0, 0, 0.5, 0.2, True, 0), (5000, 8, 400, "float16", 0, 0, 0, 0.1, False, 11),
    (5000, 8, 257, "float32", 3, 1, 0.99, 0, True, 0), (5000, 13, 512, "bfloat16", 0, 0, 0, 0, True, 0), (4100, 64, 300, "float32", 0, 0, 0.8, 0, False, 0)]


@pytest.mark.parametrize("N,k,E,dtype,step,shift,masked,padded,biased,few", CASES)
def test_many_tokens(N, k, E, dtype, step, shift, masked, padded, biased, few):
    whole_check(N, k, E, dtype, step, shift, masked, padded, biased, few)

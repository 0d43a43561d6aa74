"""Products with 4-bit weights (gemv_ar_q4_*) for values of x that a model has
and a normal distribution does not, in the kernel for few rows and in the
matrix-product kernel.

Inputs are whole multiples of a power of two, scales powers of two, and sums
below 2^24 of their common unit leave fp32 nothing to round: results in fp32
are compared bit for bit."""
import numpy as np
import pytest

from tests.test_gpu_q4 import TYPES, Weights, _abi

pytestmark = pytest.mark.gpu

# rows, M, group: the kernel for few rows, and the matrix-product kernel with 32 and 64 rows of x to a tile
LAUNCHES = [(16, 4100, 128), (400, 4100, 128), (1000, 4100, 128), (16, 8200, 64), (1000, 8200, 64), (1000, 8200, 32)]


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    torch.cuda.set_device(0)
    yield
    torch.cuda.synchronize()


def _forward(w, x, M, K, group, dtype, y_dtype="float32", glu=0):
    import torch
    import paper_2305_06942_amd as ebag
    plan = ebag.Q4Gemv(M, K, group, _abi(dtype), glu=glu)
    y = torch.full((x.shape[0], M // 2 if glu else M), float("nan"), dtype=getattr(torch, y_dtype), device="cuda")
    plan.forward(w.codes, w.scales, w.zeros, x, y)
    torch.cuda.synchronize()
    plan.close()
    return y


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("rows,M,group", LAUNCHES)
def test_large_values_of_one_sign(rows, M, group, zeros, dtype):
    """x from 512 to 59904, all positive: finite in fp16, whose range ends at
    65504, where the sum of 32 of them does not stay.  In units of 512 / 8 a
    result is below 15 * 16 * 117 * 260 < 2^23."""
    import torch
    rng = np.random.default_rng([71, rows, group])
    K = 260
    w = Weights(rng, 1, M, K, group, dtype, zeros, exact=True, at=0)
    x64 = 512.0 * rng.integers(1, 118, size=(rows, K))
    y = _forward(w, torch.from_numpy(x64).to(getattr(torch, dtype)).cuda(), M, K, group, dtype)
    assert np.array_equal(y.double().cpu().numpy(), x64 @ w.w64[0].T)

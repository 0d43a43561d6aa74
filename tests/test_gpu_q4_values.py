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


@pytest.mark.parametrize("K,dtype", [((1 << 31) - 4097, "float16"), ((1 << 31) - 4099, "bfloat16")])
def test_the_longest_rows(K, dtype):
    """The most columns there may be: x is staged in parts, the last of which
    ends behind 2^31.  A thousand columns of x are not zero, the last ones
    among them; whole numbers below 2^24."""
    import torch
    import paper_2305_06942_amd as ebag
    M, group = 2, 1 << 30
    rng = np.random.default_rng(72)
    codes = torch.randint(0, 256, (1, M, (K + 1) // 2), dtype=torch.uint8, device="cuda")
    scales = torch.tensor([[[1.0, 2.0], [0.5, 1.0]]], dtype=getattr(torch, dtype), device="cuda")
    at = np.unique(np.concatenate([rng.integers(0, K, size=980), np.arange(K - 10, K), [0, group - 1, group, 2 * group - 5000]]))
    values = rng.integers(-9, 10, size=len(at)).astype(np.float64)
    cols = torch.from_numpy(at).cuda()
    x = torch.zeros((1, K), dtype=scales.dtype, device="cuda")
    x[0, cols] = torch.from_numpy(values).to(x.dtype).cuda()
    y = torch.full((1, M), float("nan"), device="cuda")
    plan = ebag.Q4Gemv(M, K, group, _abi(dtype))
    plan.forward(codes, scales, None, x, y)
    byte = codes[0][:, cols // 2].cpu().numpy()
    q = np.where(at % 2, byte >> 4, byte & 15) - 8.0
    want = (q * scales[0].double().cpu().numpy()[:, at // group]) @ values
    assert np.array_equal(y[0].double().cpu().numpy(), want)
    plan.close()
    del codes, x
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("group", [32, 128])
@pytest.mark.parametrize("K", [1, 3, 6, 8, 13, 20, 27, 30, 31, 33])
def test_many_rows_of_few_columns(K, group, dtype):
    """Rows of codes of one to seventeen bytes in the matrix-product kernel, at
    every distance from a multiple of 4, the last one at its allocation's end."""
    import torch
    rng = np.random.default_rng([73, K, group])
    rows, M = 1000, 8199
    x64 = rng.integers(-9, 10, size=(rows, K)).astype(np.float64)
    x = torch.from_numpy(x64).to(getattr(torch, dtype)).cuda()
    for at in range(4):
        w = Weights(rng, 1, M, K, group, dtype, True, exact=True, at=at)
        y = _forward(w, x, M, K, group, dtype)
        want = torch.from_numpy(x64).cuda() @ torch.from_numpy(np.ascontiguousarray(w.w64[0].T)).cuda()
        assert torch.equal(y.double(), want), at

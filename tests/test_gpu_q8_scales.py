"""Products in 8-bit integers with scales of every size: the sum, exact and rounded to fp32, times the fp32 product of the two
scales, as the definition has it, bit for bit in every kernel: where that product is below 2^-126, or an infinity, too."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

TYPES = ("float32", "float16", "bfloat16")


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    torch.cuda.set_device(0)
    yield
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,M,K", [(1, 300, 304), (3, 300, 304), (40, 301, 1000), (200, 2000, 130), (1500, 1030, 260), (4000, 2100, 130)])
def test_scales_of_every_size(rows, M, K, dtype):
    import torch
    import paper_2305_06942_amd as ebag
    rng = np.random.default_rng([121, rows, M])
    plan = ebag.Q8Gemv(M, K, TYPES.index(dtype))
    codes = torch.from_numpy(rng.integers(-127, 128, size=(1, M, plan.pitch)).astype(np.int8)).cuda()
    codes[0, ::7] = 0  # sums of zero
    most = 12 if dtype == "float16" else 110
    scales = (rng.uniform(0.5, 1, size=(1, M)) * 2.0 ** rng.integers(-140, 120, size=(1, M))).astype(np.float32)
    x = rng.standard_normal((rows, K)) * 2.0 ** rng.integers(-most, most, size=(rows, 1))
    x = torch.from_numpy(x).to(getattr(torch, dtype)).cuda()
    xq, xs = torch.empty((rows, plan.pitch), dtype=torch.int8, device="cuda"), torch.empty(rows, device="cuda")
    plan.round(x, xq, xs)
    sums = xq[:, :K].double().cpu().numpy() @ codes[0, :, :K].double().cpu().numpy().T
    with np.errstate(all="ignore"):
        want = sums.astype(np.float32) * (xs.cpu().numpy()[:, None] * scales)
    y = torch.full((rows, M), 7.0, device="cuda")
    plan.forward(codes, torch.from_numpy(scales).cuda(), x, y, xq, xs)
    got = y.cpu().numpy()
    bad = np.argwhere(~((got == want) | (np.isnan(got) & np.isnan(want))))
    assert not len(bad), (len(bad), bad[0], got[tuple(bad[0])], want[tuple(bad[0])])
    plan.close()

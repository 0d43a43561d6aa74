"""One row on a 16-byte boundary, which the product rounds itself: every instance of that kernel, matrices and rows up to the
largest that it takes and the next ones, against 64 bits and against the row rounded first; bounds as in test_gpu_q8.py."""
import numpy as np
import pytest

from tests.test_gpu_q8 import Weights, _check, _plan, _rounded, _scratch, _strided, _untouched, _want

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    torch.cuda.set_device(0)
    yield
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("M,K,glu", [
    (4096, 1024, 0), (5, 8, 0), (300, 512, 1), (300, 1048, 1), (7000, 136, 0), (7000, 2000, 0), (13000, 64, 1), (13000, 1000, 1), (48, 12288, 0), (16384, 96, 0),
    (16400, 96, 0), (32768, 160, 1), (32770, 160, 1), (33, 16384, 0), (34, 19200, 1), (17, 19456, 0), (40, 32640, 1), (17, 32768, 0)])
def test_one_row(M, K, glu, dtype):
    import torch
    rng = np.random.default_rng([131, M, K])
    plan = _plan(M, K, dtype, glu=glu)
    w = Weights(rng, plan, M, K)
    x = torch.from_numpy(rng.standard_normal((1, K))).to(getattr(torch, dtype)).cuda()
    xq64, xs64 = _rounded(x.double().cpu().numpy())
    want, b = _want(xq64, xs64.astype(np.float64), w, 0, glu)
    xq, xs = _scratch(plan, 1)
    for y_dtype in {dtype, "float32"}:
        y, buf = _strided(1, plan.wide, y_dtype, 0, 3)
        plan.forward(w.codes, w.scales, x, y, xq, xs)
        _check(y, want, b, y_dtype)
        _untouched(buf, 1, plan.wide, 0, 3)
        plan.round(x, xq, xs)
        first = torch.full_like(y, float("nan"))
        plan.forward(w.codes, w.scales, None, first, xq, xs)
        assert torch.equal(first, y), "another result than of the row rounded first"
    plan.close()

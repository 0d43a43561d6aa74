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


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,M,group", LAUNCHES)
def test_fp32_results_are_as_near_as_an_fp32_product(rows, M, group, dtype):
    """4096 columns of normal x: the root mean square distance from the result in
    64 bits is at most twice that of the same product in fp32 by torch; and no
    result is further off than the sum of |weight * x|, whose terms are exact,
    times 2^-23 for each of at most 128 products of a group in a chain, a
    multiply-add per 32 columns and 16 partial sums."""
    import torch
    rng = np.random.default_rng([74, rows, group])
    K = 4096
    w = Weights(rng, 1, M, K, group, dtype, True, at=0)
    x = torch.from_numpy(rng.standard_normal((rows, K))).to(getattr(torch, dtype)).cuda()
    y = _forward(w, x, M, K, group, dtype).double()
    w64 = torch.from_numpy(np.ascontiguousarray(w.w64[0].T)).cuda()
    want = x.double() @ w64
    far = (y - want).abs()
    assert bool((far <= (144 + K / 16) * 2.0 ** -23 * (x.double().abs() @ w64.abs())).all())
    plain = x.float() @ w64.float()
    rms = lambda v: float(v.square().mean().sqrt())  # noqa: E731
    assert rms(far) <= 2 * rms(plain.double() - want), (rms(far), rms(plain.double() - want))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,M", [(3, 512), (1000, 8200)])
def test_silu_in_fp32(rows, M, dtype):
    """One column of x is 1, the gates are a scale times -8 .. 7, rounded to fp32 where
    the scale has 24 bits, and the up weights 1, so y is silu of a known number.  An exponential good to one unit in the
    last place (2^-23), 1 + e, a division and two products of 2^-24 each make
    2^-21; an exponential below 2^-126 is off by 2^-149, times |gate| below 128."""
    import torch
    rng = np.random.default_rng([75, rows])
    K = group = 32
    w = Weights(rng, 1, M, K, group, dtype, False, at=0)
    half = M // 2
    scales = torch.empty((1, M, 1), dtype=torch.float64)
    scales[0, :half, 0] = torch.from_numpy(np.concatenate([np.linspace(0.01, 13, half - 56), 12.99 - np.linspace(0, 2, 56)]))
    scales[0, half:] = 1
    w.scales = scales.to(getattr(torch, dtype)).cuda()
    w.codes[0, half:] = 0x99
    x = torch.zeros((rows, K), dtype=w.scales.dtype, device="cuda")
    x[:, 0] = 1
    y = _forward(w, x, M, K, group, dtype, glu=1).double().cpu().numpy()
    g = (w.scales[0, :half, 0].double().cpu().numpy() * ((w.codes[0, :half, 0].cpu().numpy() & 15) - 8.0)).astype(np.float32).astype(np.float64)
    want = g * np.where(g < 0, np.exp(-np.abs(g)), 1.0) / (1 + np.exp(-np.abs(g)))
    assert g.min() < -90 and g.max() > 80
    assert np.all(np.abs(y - want) <= 2.0 ** -21 * np.abs(want) + 128 * 2.0 ** -149)


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("rows,M,group", LAUNCHES)
def test_every_bit_of_fp32_x_counts(rows, M, group, zeros):
    """One column of each row of x is not zero and has 24 bits; the weight there is
    a power of two times a code less its zero point that is one, too: the
    product is known bit for bit, whatever the other columns' weights are."""
    import torch
    rng = np.random.default_rng([76, rows, group])
    K = 260
    w = Weights(rng, 1, M, K, group, "float32", zeros, exact=True, at=0)
    at = rng.integers(0, K, size=rows)
    significand = rng.integers(1 << 23, 1 << 24, size=rows) | 1
    v = np.where(rng.random(rows) < 0.5, -1.0, 1.0) * significand * 2.0 ** rng.integers(-60, 60, size=rows)
    x = torch.zeros((rows, K), device="cuda")
    x[torch.arange(rows), torch.from_numpy(at).cuda()] = torch.from_numpy(v.astype(np.float32)).cuda()
    y = _forward(w, x, M, K, group, "float32").double().cpu().numpy()
    weight = w.w64[0][:, at].T  # [rows, M]
    m, _ = np.frexp(np.abs(weight))
    known = (m == 0.5) | (weight == 0)
    assert known.mean() > 0.2
    assert np.array_equal(y[known], (weight * v[:, None])[known])
    # Others: (q - zero) x of up to 28 bits is rounded to 24 once by each of three additions.
    assert np.all(np.abs(y - weight * v[:, None]) <= 3 * 2.0 ** -23 * np.abs(weight * v[:, None]))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("y32", [False, True])
@pytest.mark.parametrize("rows,M,group", LAUNCHES)
def test_rows_are_their_own(rows, M, group, y32, dtype):
    """Every row's result is the same bits whatever the other rows hold; a row
    with an infinity or NaN has no finite result."""
    import torch
    rng = np.random.default_rng([77, rows, group])
    K = 500
    w = Weights(rng, 1, M, K, group, dtype, True, at=0)
    x = torch.from_numpy(rng.standard_normal((rows, K))).to(getattr(torch, dtype)).cuda()
    y_dtype = "float32" if y32 else dtype
    clean = _forward(w, x, M, K, group, dtype, y_dtype)
    bad = np.unique(np.concatenate([[0, rows - 1], rng.integers(0, rows, size=rows // 5)]))
    value = torch.tensor([float("inf"), float("-inf"), float("nan")], dtype=x.dtype, device="cuda")
    x[torch.from_numpy(bad).cuda(), torch.from_numpy(rng.integers(0, K, size=len(bad))).cuda()] = value[torch.arange(len(bad), device="cuda") % 3]
    dirty = _forward(w, x, M, K, group, dtype, y_dtype)
    good = torch.ones(rows, dtype=torch.bool, device="cuda")
    good[torch.from_numpy(bad).cuda()] = False
    assert torch.equal(clean[good], dirty[good])
    assert not torch.isfinite(dirty[~good]).any()

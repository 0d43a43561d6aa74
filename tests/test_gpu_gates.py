"""silu(gate) * up over the whole range of gates, in every kernel that has it, against 64 bits.

A gate g is one weight's code times its row's x, so its sum has no error and g is off by
two roundings at most; 4 u |g| with u = 2^-24 covers it.  Where g < 0, ln|silu| moves
by at most (1 + 1 / |g|) times that, where g > 0 by 1.3 / g times: below (|g| + 2) 4 u of
the result.  With an exponential good to (|g| + 8) 2^-22 for a 16-bit y and the full one
below that, rel = (2 |g| + 10) 2^-22 is the relative distance of silu(g).  As an fp32 number silu
is off by 2^-149 besides; an fp32 y's exponential below 2^-126 is off by as much itself, times
|g|, of which 128 is the most with a result: `floor`.  up has two roundings, the product one: 5 u.
Rounding keeps order, so a result lies between want - b and want + b, both rounded."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

TYPES = ("float32", "float16", "bfloat16")
U = 2.0 ** -24
GATES = np.concatenate((np.linspace(-130, 130, 521), [-1e30, -1e10, -1e3, -200, -103.9, -104.1, -88.73, -88.72, -87.34, -87.33, -64.01, -63.99,
                                                      -1e-3, -1e-30, 0, 1e-30, 1e-3, 17, 19.99, 20.01, 64.01, 88.73, 200, 1e3, 1e10, 1e30]))


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    torch.cuda.set_device(0)
    yield
    torch.cuda.synchronize()


def _check(got, g, u, y_dtype, off=4):
    """off: how far g and u may be from the numbers themselves, in u."""
    import torch
    e = np.exp(-np.abs(g))
    act = g * np.where(g < 0, e, 1.0) / (1 + e)
    floor = (128 if y_dtype == "float32" else 1) * 2.0 ** -149
    rel = (np.abs(g) + 8) * 2.0 ** -22 + (np.abs(g) + 2) * off * U
    b = 1.01 * (np.abs(act) * rel + floor) * np.abs(u) + (off + 1) * U * np.abs(act * u) + 2.0 ** -149
    want = act * u
    got = got.double().cpu().numpy()
    lo, hi = (torch.from_numpy(v).to(getattr(torch, y_dtype)).double().numpy() for v in (want - b, want + b))
    ok = (lo <= got) & (got <= hi)
    assert np.all(ok), (f"{int((~ok).sum())} of {ok.size} outside, gates {g[~ok].min()} to {g[~ok].max()}, the first at "
                        f"{np.argwhere(~ok)[0]}, gate {g[~ok][0]}, up {u[~ok][0]}: {got[~ok][0]} not in [{lo[~ok][0]}, {hi[~ok][0]}]")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,experts", [(1, 1), (3, 1), (70, 1), (300, 1), (1500, 1), (6, 3), (900, 3)])
def test_gates_in_8_bits(rows, experts, dtype):
    import torch
    import paper_2305_06942_amd as ebag
    rng = np.random.default_rng([111, rows, experts])
    K = 8
    gates, ups = np.repeat(GATES, 4), np.tile([1.0, -3e-4, 1e6, 1e30], len(GATES))
    H = len(gates)
    plan = ebag.Q8Gemv(2 * H, K, TYPES.index(dtype), experts=experts, glu=1)
    codes = torch.from_numpy(rng.integers(-127, 128, size=(experts, 2 * H, plan.pitch)).astype(np.int8)).cuda()
    first = torch.from_numpy(np.where(np.concatenate((gates, ups)) < 0, -127, 127).astype(np.int8)).cuda()
    codes[:, :, 0] = first
    scales = torch.from_numpy((np.abs(np.concatenate((gates, ups))) / 127).astype(np.float32)).cuda().expand(experts, -1).contiguous()
    x = torch.zeros((rows, K), dtype=getattr(torch, dtype), device="cuda")
    x[:, 0] = torch.from_numpy(rng.choice([1.0, 1.0, 0.5, 0.96875, 0.25], size=rows))
    x[rows - 1, 0] = 1
    xq, xs = torch.empty((rows, plan.pitch), dtype=torch.int8, device="cuda"), torch.empty(rows, device="cuda")
    plan.round(x, xq, xs)
    sums = 127.0 * first.double().cpu().numpy()
    z = sums[None] * xs.double().cpu().numpy()[:, None] * scales[0].double().cpu().numpy()[None]
    for y_dtype in {dtype, "float32"}:
        y = torch.full((rows, H), float("nan"), dtype=getattr(torch, y_dtype), device="cuda")
        if experts == 1:
            plan.forward(codes, scales, x, y, xq, xs)
        else:
            ends = torch.tensor([0, rows // 3, rows // 3, rows], dtype=torch.int32, device="cuda")
            plan.experts(codes, scales, x, ends, y, xq, xs)
        _check(y, z[:, :H], z[:, H:], y_dtype)
    plan.close()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,experts", [(1, 1), (5, 1), (40, 1), (1000, 1), (900, 3)])
def test_gates_in_4_bits(rows, experts, dtype):
    """One column of x is not zero, and its weight 7 times the scale.  A sum is made of that term with a part of up to 143 s |x| that
    comes off again: four roundings of 286 s |x| 2^-23, of 7 s |x| less than 330 u."""
    import torch
    import paper_2305_06942_amd as ebag
    rng = np.random.default_rng([112, rows, experts])
    K = 32
    most = 1e3 if dtype == "float16" else 1e30
    gates = GATES[(np.abs(GATES) <= most) & ((np.abs(GATES) >= 1e-3) | (dtype != "float16"))]
    gates, ups = np.repeat(gates, 4), np.tile([1.0, -3e-2, 1e4, most], len(gates))
    H = len(gates)
    plan = ebag.Q4Gemv(2 * H, K, K, TYPES.index(dtype), experts=experts, glu=1)
    codes = torch.from_numpy(rng.integers(0, 256, size=(experts, 2 * H, K // 2), dtype=np.uint8)).cuda()
    sign = np.sign(np.concatenate((gates, ups)))
    codes[:, :, 0] = torch.from_numpy((8 + 7 * sign).astype(np.uint8)).cuda()
    scales = torch.from_numpy(np.abs(np.concatenate((gates, ups))) / 7).to(getattr(torch, dtype)).cuda()
    x = torch.zeros((rows, K), dtype=scales.dtype, device="cuda")
    x[:, 0] = torch.from_numpy(rng.choice([1.0, 1.0, 0.5, 0.96875, 0.25], size=rows))
    x[rows - 1, 0] = 1
    z = x[:, :1].double().cpu().numpy() * (7 * sign * scales.double().cpu().numpy())[None]
    weights = codes, scales.expand(experts, -1).contiguous(), None
    for y_dtype in {dtype, "float32"}:
        y = torch.full((rows, H), float("nan"), dtype=getattr(torch, y_dtype), device="cuda")
        if experts == 1:
            plan.forward(*weights, x, y)
        else:
            ends = torch.tensor([0, rows // 3, rows // 3, rows], dtype=torch.int32, device="cuda")
            plan.experts(*weights, x, ends, y)
        _check(y, z[:, :H], z[:, H:], y_dtype, 330)
    plan.close()

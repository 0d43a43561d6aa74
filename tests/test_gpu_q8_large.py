"""Products in 8-bit integers of more tiles than one launch of the fastest kernel has threads for."""
import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    torch.cuda.set_device(0)
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


def _room(gib):
    import torch
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < gib << 30:
        pytest.skip(f"needs {gib} GiB of the GPU's memory")


def _within(y, xq, xs, codes, scales):
    """The sum is exact and whole, its rounding, the scales' product and the result's make 3 steps."""
    want = (xq.double() @ codes.double().t().contiguous()) * xs.double()[:, None] * scales.double()
    return bool(((y.double() - want).abs() <= want.abs() * 4 * U + 2.0 ** -149).all())


@pytest.mark.parametrize("experts", [1, 3])
def test_many_rows(experts):
    import torch
    import paper_2305_06942_amd as ebag
    _room(90)
    rows, M, K = (1 << 29) + 3, 2, 1
    plan = ebag.Q8Gemv(M, K, ebag.EBAG_BF16, experts=experts)
    codes = torch.randint(-127, 128, (experts, M, plan.pitch), dtype=torch.int8, device="cuda")
    scales = torch.rand((experts, M), device="cuda") + 0.5
    x = torch.empty((rows, K), dtype=torch.bfloat16, device="cuda").normal_()
    xq, xs = torch.empty((rows, plan.pitch), dtype=torch.int8, device="cuda"), torch.empty(rows, device="cuda")
    y = torch.full((rows, M), float("nan"), device="cuda")
    ends = [0, 1 << 28, (1 << 28) + 5, rows - 2] if experts > 1 else [0, rows]
    if experts > 1:
        plan.experts(codes, scales, x, torch.tensor(ends, dtype=torch.int32, device="cuda"), y, xq, xs)
        assert y[rows - 2:].eq(0).all()
    else:
        plan.forward(codes, scales, x, y, xq, xs)
    for e in range(experts):
        for at in range(ends[e], ends[e + 1], 1 << 24):
            n = slice(at, min(at + (1 << 24), ends[e + 1]))
            assert _within(y[n], xq[n, :K], xs[n], codes[e, :, :K], scales[e])
    for at in range(0, rows, 1 << 24):
        part = x[at:at + (1 << 24), 0].float()
        assert torch.equal(xs[at:at + (1 << 24)], (part.double().abs() / 127).float())
        assert torch.equal(xq[at:at + (1 << 24), 0].float(), 127 * part.sign())
    plan.close()


def test_many_columns_of_y():
    import torch
    import paper_2305_06942_amd as ebag
    _room(90)
    rows, M, K = 1, (1 << 29) + 6, 4
    plan = ebag.Q8Gemv(M, K, ebag.EBAG_BF16)
    codes, scales = torch.empty((1, M, plan.pitch), dtype=torch.int8, device="cuda"), torch.empty((1, M), device="cuda").uniform_(0.5, 1.5)
    for at in range(0, M, 1 << 26):
        codes[0, at:at + (1 << 26), :K].random_(-127, 128)
    x = torch.randn((rows, K), device="cuda").to(torch.bfloat16)
    xq, xs = torch.empty((rows, plan.pitch), dtype=torch.int8, device="cuda"), torch.empty(rows, device="cuda")
    y = torch.full((rows, M), float("nan"), device="cuda")
    plan.forward(codes, scales, x, y, xq, xs)
    for at in range(0, M, 1 << 23):
        m = slice(at, at + (1 << 23))
        assert _within(y[:, m], xq[:, :K], xs, codes[0, m, :K], scales[0, m])
    plan.close()

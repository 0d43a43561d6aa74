"""Tokens by expert (ebag_a2a_moe_*) at values and widths where an operator's
vectors can go wrong."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    torch.cuda.set_device(0)
    yield
    torch.cuda.synchronize()


def _plan_of(N, k, E, seed):
    import torch
    import paper_2305_06942_amd as ebag
    g = torch.Generator(device="cuda").manual_seed(seed)
    ids = torch.randint(0, E, (N, k), generator=g, device="cuda", dtype=torch.int32)
    plan = ebag.MoePerm(N, k, E)
    offsets = torch.empty(E + 1, dtype=torch.int32, device="cuda")
    pos, src = torch.empty_like(ids), torch.empty(N * k, dtype=torch.int32, device="cuda")
    plan.sort(ids, offsets, pos, src)
    return plan, offsets, pos


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("D", [5, 9, 15, 33, 250, 519, 1021, 1999, 4101])
def test_an_infinity_in_any_column_of_dout_is_an_infinite_gradient(D, dtype):
    """Token n's dout is infinite in one column, of the last twenty or so, and
    ys are powers of two with both signs: dweights is the infinity with the
    sign of ys there, and a finite sum for the last token, which has none."""
    import torch
    N, k = 24, 3
    plan, offsets, pos = _plan_of(N, k, 4, D)
    t = getattr(torch, dtype)
    g = torch.Generator(device="cuda").manual_seed(D)
    ys = (torch.randint(0, 2, (N * k, D), generator=g, device="cuda") * 2.0 - 1.0).to(t)
    dout = torch.ones((N, D), device="cuda", dtype=t)
    at = [max(0, D - 1 - n) for n in range(N - 1)]
    for n, c in enumerate(at):
        dout[n, c] = float("inf")
    w = torch.ones((N, k), device="cuda")
    dys, dw = torch.empty_like(ys), torch.empty_like(w)
    plan.combine_backward(dout, ys, offsets, pos, w, dys, dw)
    rows = ys[pos.long()].float()
    for n, c in enumerate(at):
        assert torch.equal(dw[n], rows[n, :, c] * float("inf")), (n, c, dw[n])
    assert torch.equal(dw[N - 1], rows[N - 1].sum(1))
    plan.close()


@pytest.mark.parametrize("D", [(1 << 29) - 1, (1 << 29) - 3, (1 << 29) - 4])
def test_the_widest_rows(D):
    """fp32 rows of just under 2^31 bytes, the most there may be: every column
    is moved, the last ones too.  ys are +-1 and -+1 in turn and dout 1 in eight
    columns only, so the dot product is a whole number."""
    import torch
    plan, offsets, pos = _plan_of(1, 1, 1, 0)
    x = torch.zeros((1, D), device="cuda")
    at = torch.tensor([0, 1, 2, D // 2, D - 4, D - 3, D - 2, D - 1], device="cuda")
    values = torch.arange(1.0, 9.0, device="cuda")
    x[0, at] = values
    y = torch.full_like(x, float("nan"))
    plan.dispatch(x, offsets, pos, y)
    assert torch.equal(x, y)
    w = torch.full((1, 1), 2.0, device="cuda")
    y.fill_(float("nan"))
    plan.combine(x, offsets, pos, w, y)
    assert torch.equal(y, x * 2)
    y.fill_(float("nan"))
    plan.dispatch_backward(x, offsets, pos, y)
    assert torch.equal(y, x)
    ys = torch.ones_like(x)
    ys[0, 1::2] = -1.0
    y.fill_(float("nan"))
    dw = torch.full_like(w, float("nan"))
    plan.combine_backward(x, ys, offsets, pos, w, y, dw)
    assert torch.equal(y, x * 2)
    assert float(dw) == float((values * ys[0, at]).sum())
    plan.close()
    del x, y, ys
    torch.cuda.empty_cache()

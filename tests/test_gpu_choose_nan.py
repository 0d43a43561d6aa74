"""Tokens without a number among their logits do not count: the router's results are those of the other tokens alone."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    torch.cuda.set_device(0)
    yield
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("normalise", [True, False])
@pytest.mark.parametrize("N,k,E", [(40, 3, 6), (300, 8, 128), (20000, 8, 128), (20000, 2, 100), (9000, 12, 300)])
def test_tokens_of_nan_alone_do_not_count(N, k, E, normalise, dtype):
    """Beside the same call with those tokens masked as a whole: the same bits."""
    import torch
    import paper_2305_06942_amd as ebag
    plan = ebag.MoePerm(N, k, E)
    logits = torch.randn((N, E), device="cuda").to(getattr(torch, dtype))
    bad = torch.zeros(N, dtype=torch.bool, device="cuda")
    bad[N - N // 5:] = True
    empty = logits.clone()
    logits[bad], empty[bad] = float("nan"), -float("inf")
    mixed = torch.rand((N, E), device="cuda") < 0.5
    mixed[:, 0] = False
    logits[(bad & (torch.arange(N, device="cuda") % 2 == 0))[:, None] & mixed] = -float("inf")

    def call(x):
        new = lambda *s, t=torch.float32: torch.full(s, 9, dtype=t, device="cuda")  # noqa: E731
        ids, w, counts, sums, losses = new(N, k, t=torch.int32), new(N, k), new(E + 1, t=torch.int32), new(E + 1), new(2)
        plan.choose(x, ids, w, counts, sums, losses, new(plan.choose_work), normalise=normalise)
        out = torch.full_like(x, 9)
        plan.choose_backward(x, ids, torch.ones_like(w), out, counts=counts, dlosses=torch.ones(2, device="cuda"), normalise=normalise)
        return ids, w, counts, sums, losses, out

    got, want = call(logits), call(empty)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    ids, w, counts, _, losses, out = got
    assert counts[E] == N - N // 5 and losses.isfinite().all() and (losses > 0).all()
    assert (ids[bad] == -1).all() and w[bad].eq(0).all() and out[bad].eq(0).all()
    plan.close()

"""The router where masks, choices, strides, streams and sizes are out of the ordinary; bounds as in test_gpu_choose.py."""
import numpy as np
import pytest

from tests import choose_definition as definition
from tests.test_gpu_choose import Call, _check, _np, _strided, _within

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


def _plan(N, k, E):
    import paper_2305_06942_amd as ebag
    return ebag.MoePerm(N, k, E)


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("N,k,E", [(40, 4, 7), (50, 6, 100), (5000, 8, 60)])
def test_masks_of_the_lowest_value(N, k, E, dtype):
    """The type's lowest number is a logit like any other: chosen behind all larger ones, ahead of -inf, and a row of nothing
    else has them all alike.  Such a row's squared logarithm may be no number of the type, so that loss has no gradient here."""
    import torch
    rng = np.random.default_rng([91, N, E])
    low = float(torch.finfo(getattr(torch, dtype)).min)
    v = rng.standard_normal((N, E))
    v[rng.random((N, E)) < 0.5] = low
    v[rng.random((N, E)) < 0.3] = -np.inf
    v[::5] = low
    v[1::5] = np.where(rng.random((len(v[1::5]), E)) < 0.5, low, -np.inf)
    v[2::5] = -np.inf
    v[3::5, 1:] = low
    logits = _strided(N, E, dtype, 0, 0, v)[0]
    plan = _plan(N, k, E)
    for normalise in (True, False):
        call = Call(plan, logits, k, E, False, normalise=normalise)
        row, ids = _check(call, logits, k, E, None, None, normalise)
        whole = Call(plan, logits, k, E, True, normalise=normalise)
        with np.errstate(over="ignore"):
            counts, sums, err, losses, losses_err = definition.totals(row, ids, E, 400 + N // 256)
        assert np.array_equal(whole.counts.cpu().numpy(), counts) and torch.equal(whole.ids, call.ids)
        _within(whole.sums[:-1], sums[:-1], err[:-1], what="sums")
        _within(whole.losses[:1], losses[:1], losses_err[:1], what="balance")
        dw, dl = torch.randn((N, k), device="cuda"), torch.tensor((0.5 * N, 0.0), device="cuda")
        out = torch.full_like(logits, float("nan"))
        plan.choose_backward(logits, call.ids[:N], dw, out, counts=whole.counts, dlosses=dl, normalise=normalise)
        want, b = definition.gradient(row, ids, normalise, _np(dw), counts, _np(dl))
        _within(out, want, b, dtype, "gradient")
    plan.close()


@pytest.mark.parametrize("normalise", [True, False])
@pytest.mark.parametrize("N,k,E", [(9, 4, 6), (30, 64, 5), (20, 12, 300), (9000, 3, 40)])
def test_gradient_of_ids_that_repeat_or_are_out_of_range(N, k, E, normalise):
    """Ids of the caller's own: each place counts by itself, so an expert named twice gets both parts; ones outside are none.
    Up to k parts are added up in place of one: k steps of their sizes' sum on top of the bounds."""
    import torch
    rng = np.random.default_rng([92, N, k, E])
    plan = _plan(N, k, E)
    logits = _strided(N, E, "float32", 0, 0, rng.standard_normal((N, E)))[0]
    ids = rng.integers(0, E, size=(N, k)).astype(np.int32)
    ids[rng.random((N, k)) < 0.2] = -1
    ids[0] = ids[0, 0] if ids[0, 0] >= 0 else 0
    given = ids.copy()
    given[(ids < 0) & (rng.random((N, k)) < 0.7)] = rng.choice([-2 ** 31, -2, E, E + 1, 511, 2 ** 31 - 1])
    given[(given >= 0) & (given < E) & (ids < 0)] = -1
    dw = torch.from_numpy(rng.standard_normal((N, k)).astype(np.float32)).cuda()
    out = torch.full_like(logits, float("nan"))
    plan.choose_backward(logits, torch.from_numpy(given).cuda(), dw, out, normalise=normalise)
    row = definition.Row(_np(logits))
    want, b = definition.gradient(row, ids, normalise, _np(dw), None, None)
    w, d = definition.weights(row, ids, normalise)[0], np.where(ids >= 0, np.abs(_np(dw)), 0.0)
    size = np.zeros((N, E))
    rows, places = np.nonzero(ids >= 0)
    np.add.at(size, (rows, ids[rows, places]), (w * (d + (w * d).sum(1, keepdims=True)))[rows, places])
    _within(out, want, b + k * U * size, what="gradient")
    plan.close()


def test_live_is_any_number_but_zero():
    import torch
    N, k, E = 70, 2, 9
    plan = _plan(N, k, E)
    logits = torch.randn((N, E), device="cuda")
    live = torch.tensor([0, 1, 2, 128, 255] * 14, dtype=torch.uint8, device="cuda")
    call = Call(plan, logits, k, E, True, None, live)
    same = Call(plan, logits, k, E, True, None, live.bool())
    assert all(torch.equal(a.nan_to_num(7), b.nan_to_num(7)) for a, b in zip(call.outputs(), same.outputs()))
    assert (call.ids[:N][live == 0] == -1).all() and (call.ids[:N][live > 0] >= 0).all()
    plan.close()


def test_two_streams_at_once():
    """Calls of one plan that run at the same time, with memory of their own."""
    import torch
    N, k, E = 20000, 8, 256
    plan = _plan(N, k, E)
    streams = [torch.cuda.Stream() for _ in range(2)]
    logits = [torch.randn((N, E), device="cuda") for _ in range(2)]
    calls = [Call(plan, x, k, E) for x in logits]
    want = [c.outputs() for c in calls]
    for c in calls:
        for t in (c.ids, c.weights, c.counts, c.sums, c.losses):
            t.fill_(-5)
    torch.cuda.synchronize()
    for _ in range(10):
        for c, x, s in zip(calls, logits, streams):
            plan.choose(x, c.ids[:N], c.weights[:N], c.counts, c.sums, c.losses, c.work, stream=s)
    torch.cuda.synchronize()
    for c, w in zip(calls, want):
        assert torch.equal(c.ids[:N], w[0][:N]) and torch.equal(c.weights[:N], w[1][:N])
        assert all(torch.equal(a, b) for a, b in zip(c.outputs()[2:], w[2:]))
    plan.close()


def test_rows_far_apart():
    """Offsets of rows behind 2^32 bytes."""
    import torch
    N, k, E, step = 700, 3, 20, 1 << 22
    plan = _plan(N, k, E)
    wide = torch.empty((N, step), dtype=torch.bfloat16, device="cuda")
    near = torch.randn((N, E), device="cuda").to(torch.bfloat16)
    wide[:, :E] = near
    a, b = Call(plan, wide[:, :E], k, E), Call(plan, near, k, E)
    assert all(torch.equal(x.nan_to_num(7), y.nan_to_num(7)) for x, y in zip(a.outputs(), b.outputs()))
    dw, dl = torch.randn((N, k), device="cuda"), torch.tensor((1.0, 2.0), device="cuda")
    out = torch.empty_like(near)
    plan.choose_backward(near, b.ids[:N], dw, out, counts=b.counts, dlosses=dl)
    plan.choose_backward(wide[:, :E], b.ids[:N], dw, wide[:, 64:64 + E], counts=b.counts, dlosses=dl)
    assert torch.equal(wide[:, 64:64 + E], out) and torch.equal(wide[:, :E], near)
    plan.close()


def test_more_tokens_than_one_launch_has_threads_for():
    """2^30 tokens and a few, four lanes each; one expert, so p = 1, the logarithm is the logit, and with dlosses[1] = T / 2
    the gradient is it, too: off by roundings in fp32 and one to the type, below 2^-8 of it."""
    import torch
    N = (1 << 30) + 5
    plan = _plan(N, 1, 1)
    logits = torch.empty((N, 1), dtype=torch.bfloat16, device="cuda").normal_()
    logits[::1000001] = -float("inf")
    logits[-1] = 3.0
    none = logits == -float("inf")
    ids, weights = torch.full((N, 1), -77, dtype=torch.int32, device="cuda"), torch.full((N, 1), float("nan"), device="cuda")
    T = N - int(none.sum())
    for totals in (False, True):
        new = lambda n, t=torch.float32: torch.empty(n, dtype=t, device="cuda")  # noqa: E731
        extra = (new(2, torch.int32), new(2), new(2), new(plan.choose_work)) if totals else ()
        plan.choose(logits, ids, weights, *extra)
        assert bool((ids == torch.where(none, -1, 0)).all()) and bool((weights == torch.where(none, 0.0, 1.0)).all())
        ids.fill_(-77)
        weights.fill_(float("nan"))
    counts, sums, losses, _ = extra
    assert counts.tolist() == [T, T]
    chain = (-(-N // (256 * 256)) + 300) * U
    assert abs(float(sums[0]) - T) <= chain * T and abs(float(losses[0]) - 1) <= (chain + 8 * U)
    out = torch.full_like(logits, float("nan"))
    plan.choose_backward(logits, ids, None, out, counts=counts, dlosses=torch.tensor((0.0, T / 2), device="cuda"))
    assert bool((out[none] == 0).all())
    out.masked_fill_(none, 0)
    logits.masked_fill_(none, 0)
    for at in range(0, N, 1 << 28):
        x, y = logits[at:at + (1 << 28)].float(), out[at:at + (1 << 28)].float()
        assert bool(((x - y).abs() <= x.abs() * 2.0 ** -8).all())
    plan.close()


@pytest.mark.parametrize("N,k,E,dtype,masked,few", [
    (33000, 16, 60, "bfloat16", 0.0, 5), (17000, 9, 100, "float32", 0.9, 0), (8300, 12, 256, "float16", 0.0, 9), (4200, 16, 500, "float32", 0.3, 0),
    (8300, 17, 250, "float32", 0.0, 0), (8300, 2, 250, "bfloat16", 0.0, 4), (70000, 11, 33, "float32", 0.0, 0)])
def test_many_tokens_of_many_choices(N, k, E, dtype, masked, few):
    import torch
    from tests.test_gpu_choose import _logits
    rng = np.random.default_rng([93, N, k, E])
    plan = _plan(N, k, E)
    logits = _logits(rng, N, E, dtype, masked, 2.0, few)
    for normalise, totals in ((True, True), (False, False)):
        call = Call(plan, logits, k, E, totals, normalise=normalise)
        _check(call, logits, k, E, None, None, normalise)
    plan.close()

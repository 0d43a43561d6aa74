"""The router (ebag_a2a_moe_choose and its gradient) against the definition in 64
bits (choose_definition.py, which derives the bounds).  Choices and counts are whole
numbers and compared exactly.  Rounding to the logits' type keeps order, so a
gradient lies between want - b and want + b, both rounded to it."""
import numpy as np
import pytest

from tests import choose_definition as definition

pytestmark = pytest.mark.gpu

TYPES = ("float32", "float16", "bfloat16")


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    torch.cuda.set_device(0)
    yield
    torch.cuda.synchronize()


def _strided(rows, cols, dtype, step, shift, values=None):
    """A [rows, cols] view with cols + step elements between rows, `shift` behind its allocation's start, which holds NaN."""
    import torch
    buf = torch.full((rows * (cols + step) + shift + 16,), float("nan"), dtype=getattr(torch, dtype), device="cuda")
    view = buf[shift:shift + rows * (cols + step)].view(rows, cols + step)[:, :cols]
    if values is not None:
        view.copy_(torch.from_numpy(values).to(getattr(torch, dtype)))
    return view, buf


def _logits(rng, N, E, dtype, masked=0.0, spread=1.0, few=0, step=0, shift=0):
    """few: so many different values, for ties."""
    v = rng.standard_normal((N, E)) * spread
    if few:
        v = rng.choice(np.linspace(-2, 2, few), size=(N, E))
        v[rng.random((N, E)) < 0.1] = -0.0
        v[rng.random((N, E)) < 0.1] = 0.0
    v[rng.random((N, E)) < masked] = -np.inf
    return _strided(N, E, dtype, step, shift, v)[0]


def _np(t):
    return t.detach().double().cpu().numpy()


def _within(got, want, b, dtype="float32", what=""):
    import torch
    got = _np(got)
    lo, hi = (torch.from_numpy(v).to(getattr(torch, dtype)).double().numpy() for v in (want - b, want + b))
    ok = (lo <= got) & (got <= hi)
    assert np.all(ok), f"{what}: {int((~ok).sum())} of {ok.size} outside, first {np.argwhere(~ok)[0]}: {got[~ok][0]} not in [{lo[~ok][0]}, {hi[~ok][0]}]"


class Call:
    """One choice with every output in memory that holds something else."""

    def __init__(self, plan, logits, k, E, totals=True, bias=None, live=None, normalise=True):
        import torch
        N = logits.shape[0]
        i32, f32 = dict(dtype=torch.int32, device="cuda"), dict(device="cuda")
        self.ids, self.weights = torch.full((N + 1, k), -77, **i32), torch.full((N + 1, k), float("nan"), **f32)
        self.counts = torch.full((E + 1,), -77, **i32) if totals else None
        self.sums = torch.full((E + 1,), float("nan"), **f32) if totals else None
        self.losses = torch.full((2,), float("nan"), **f32) if totals else None
        self.work = torch.full((plan.choose_work,), float("nan"), **f32) if totals else None
        self.again = lambda: plan.choose(logits, self.ids[:N], self.weights[:N], self.counts, self.sums, self.losses, self.work,
                                         bias=bias, live=live, normalise=normalise)
        self.again()
        self.N = N

    def outputs(self):
        return [t.clone() for t in (self.ids, self.weights, self.counts, self.sums, self.losses) if t is not None]


def _check(call, logits, k, E, bias, live, normalise):
    l = _np(logits)
    b = None if bias is None else bias.cpu().numpy()
    v = None if live is None else live.cpu().numpy()
    ids = definition.choices(l, k, b, v)
    N = call.N
    assert np.array_equal(call.ids[:N].cpu().numpy(), ids), "choices"
    assert (call.ids[N:] == -77).all() and call.weights[N:].isnan().all(), "written behind the last token"
    row = definition.Row(l, v)
    _within(call.weights[:N], *definition.weights(row, ids, normalise), what="weights")
    if call.counts is not None:
        chain = 300 + -(-N // 256)
        counts, sums, err, losses, losses_err = definition.totals(row, ids, E, chain)
        assert np.array_equal(call.counts.cpu().numpy(), counts), "counts"
        _within(call.sums, sums, err, what="sums")
        _within(call.losses, losses, losses_err, what="losses")
    return row, ids


CASES = [  # tokens, choices, experts, type, step, shift, masked, padded, bias, few
    (1, 1, 1, "float32", 0, 0, 0, 0, False, 0), (1, 2, 3, "bfloat16", 1, 1, 0, 0, False, 0), (3, 4, 4, "float16", 0, 0, 0, 0, True, 0),
    (5, 3, 2, "float32", 3, 1, 0, 0, False, 0), (32, 8, 128, "float32", 0, 0, 0, 0, False, 0), (33, 8, 127, "bfloat16", 2, 3, 0.3, 0.2, True, 0),
    (64, 64, 64, "float32", 0, 0, 0.5, 0, False, 0), (17, 64, 512, "float16", 0, 0, 0, 0, True, 0), (100, 1, 512, "float32", 5, 0, 0, 0.5, False, 0),
    (257, 6, 60, "bfloat16", 0, 0, 0.5, 0.2, True, 0), (300, 2, 8, "float32", 0, 0, 0.7, 0, False, 0), (1000, 8, 256, "float32", 0, 0, 0, 0, False, 5),
    (1000, 8, 256, "bfloat16", 0, 0, 0, 0, True, 3), (5000, 4, 17, "float16", 3, 0, 0.2, 0.1, False, 9), (9001, 6, 60, "bfloat16", 0, 0, 0.5, 0.2, True, 0),
    (12000, 8, 256, "float32", 0, 0, 0, 0, False, 0), (9000, 2, 512, "float32", 0, 0, 0, 0.3, False, 0), (40000, 1, 5, "float32", 0, 0, 0, 0, True, 0),
    (34000, 4, 64, "float16", 0, 0, 0, 0, False, 0), (700, 3, 300, "bfloat16", 0, 0, 1.0, 0, False, 0), (3000, 16, 200, "float32", 0, 0, 0, 1.0, False, 0)]


@pytest.mark.parametrize("N,k,E,dtype,step,shift,masked,padded,biased,few", CASES)
def test_choose_and_gradient(N, k, E, dtype, step, shift, masked, padded, biased, few):
    import torch
    import paper_2305_06942_amd as ebag
    rng = np.random.default_rng([71, N, k, E])
    plan = ebag.MoePerm(N, k, E)
    logits = _logits(rng, N, E, dtype, masked, 2.0, few, step, shift)
    bias = torch.from_numpy(rng.standard_normal(E).astype(np.float32)).cuda() if biased else None
    live = torch.from_numpy(rng.random(N) >= padded).cuda() if padded else None
    if padded:
        logits[~live] = float("nan")
    for normalise in (True, False):
        first = Call(plan, logits, k, E, True, bias, live, normalise)
        row, ids = _check(first, logits, k, E, bias, live, normalise)
        served = Call(plan, logits, k, E, False, bias, live, normalise)
        assert torch.equal(served.ids, first.ids) and torch.equal(served.weights[:N], first.weights[:N]), "without totals"
        before = first.outputs()
        first.again()
        assert all(torch.equal(x.nan_to_num(7), y.nan_to_num(7)) if x.is_floating_point() else torch.equal(x, y)
                   for x, y in zip(before, first.outputs())), "another result on the second run"
        dw = torch.from_numpy(rng.standard_normal((N, k)).astype(np.float32)).cuda()
        dw[first.ids[:N] < 0] = float("nan")  # of no choice: not read
        dl = torch.tensor((0.7 * N, -0.2 * N), device="cuda")
        for d, l in ((dw, dl), (dw, None), (None, dl)):
            out, buf = _strided(N, E, dtype, step, shift)
            plan.choose_backward(logits, None if d is None else first.ids[:N], d, out, counts=None if l is None else first.counts,
                                 dlosses=l, live=live, normalise=normalise)
            want, b = definition.gradient(row, ids, normalise, None if d is None else _np(d), first.counts.cpu().numpy(), None if l is None else _np(l))
            _within(out, want, b, dtype, f"gradient {d is None} {l is None}")
            outside = torch.ones_like(buf, dtype=torch.bool)
            outside[shift:shift + N * (E + step)].view(N, E + step)[:, :E] = False
            assert buf[outside].isnan().all(), "written outside the rows"
    plan.close()


@pytest.mark.parametrize("normalise", [True, False])
@pytest.mark.parametrize("N,k,E", [(6, 2, 5), (9, 3, 40)])
def test_gradient_is_that_of_the_outputs(N, k, E, normalise):
    """Against central differences of <d, weights> + <g, losses> in 64 bits with the choices held: off by the third derivative
    (below 10 times the sum of the coefficients) times h^2 / 6, and by the roundings of the difference."""
    import torch
    import paper_2305_06942_amd as ebag
    rng = np.random.default_rng([72, N, E])
    plan = ebag.MoePerm(N, k, E)
    logits = _logits(rng, N, E, "float32")
    call = Call(plan, logits, k, E, True, normalise=normalise)
    l, ids = _np(logits), call.ids[:N].cpu().numpy()
    counts = call.counts.cpu().numpy()
    d, g = rng.standard_normal((N, k)).astype(np.float32), np.array([0.6, 0.3], dtype=np.float32)

    def value(at):
        row = definition.Row(at)
        w = definition.weights(row, ids, normalise)[0]
        T = counts[-1]
        balance = E / (k * T * T) * (counts[:-1] * row.p.sum(0)).sum()
        return (w * d).sum() + g[0] * balance + g[1] * (row.lse ** 2).mean()

    h = 1e-4
    want = np.empty((N, E))
    for i in np.ndindex(N, E):
        up, down = l.copy(), l.copy()
        up[i] += h
        down[i] -= h
        want[i] = (value(up) - value(down)) / (2 * h)
    out = torch.empty_like(logits)
    plan.choose_backward(logits, call.ids[:N], torch.from_numpy(d).cuda(), out, counts=call.counts, dlosses=torch.from_numpy(g).cuda(),
                         normalise=normalise)
    size = np.abs(d).sum() + np.abs(g).sum() * (1 + np.abs(definition.Row(l).lse).max())
    row = definition.Row(l)
    b = definition.gradient(row, ids, normalise, d, counts, g)[1]
    _within(out, want, b + 10 * size * h * h / 6 + 2.0 ** -50 * size / h, what="differences")
    plan.close()


def test_values_that_are_not_numbers():
    """-inf is no choice, NaN neither, +inf the first; a token with NaN or +inf gets NaN, others do not."""
    import torch
    import paper_2305_06942_amd as ebag
    inf, nan = float("inf"), float("nan")
    E, k = 6, 3
    logits = torch.tensor([[0., 1, 2, 3, 4, 5], [nan, 1, -inf, 0, 5, 2], [-inf] * 6, [nan] * 6, [inf, 1, 2, inf, 0, 0], [3., 3, 3, 3, 3, 3],
                           [-0., 0, -0., 0, -inf, -inf], [-3e38, 3e38, -3e38, -inf, -inf, -inf], [1e-45, 0, -1e-45, 2e-45, -1e-38, 1e-38],
                           [-inf, nan, -inf, 7, nan, -inf]], device="cuda")
    N = logits.shape[0]
    # 1e-45 and 2e-45 are both 2^-149 in fp32: equal.
    want = [[5, 4, 3], [4, 5, 1], [-1] * 3, [-1] * 3, [0, 3, 2], [0, 1, 2], [0, 1, 2], [1, 0, 2], [5, 0, 3], [3, -1, -1]]
    plan = ebag.MoePerm(N, k, E)
    for normalise in (True, False):
        call = Call(plan, logits, k, E, True, normalise=normalise)
        assert call.ids[:N].cpu().tolist() == want
        w = call.weights[:N].cpu()
        bad = [4] if normalise else [1, 4, 9]
        for n in range(N):
            assert w[n].isnan().any() == (n in bad), n
        assert w[2].eq(0).all() and w[3].eq(0).all() and w[5].sub(1 / 3 if normalise else 1 / 6).abs().max() < 2e-7
        assert call.counts[E] == 8
        out = torch.full_like(logits, 9.0)
        plan.choose_backward(logits, call.ids[:N], torch.ones(N, k, device="cuda"), out, normalise=normalise)
        assert out[[2, 3]].eq(0).all()
        assert out[[0, 5, 6, 7, 8]].isfinite().all()
    plan.close()


def test_bias_decides_and_leaves_the_weights():
    import torch
    import paper_2305_06942_amd as ebag
    inf = float("inf")
    logits = torch.tensor([[0., 1, 2, 3, 4]], device="cuda").repeat(3, 1)
    plan = ebag.MoePerm(3, 2, 5)
    bias = torch.tensor([inf, 0, 0, 0, -inf], device="cuda")
    call = Call(plan, logits, 2, 5, True, bias=bias, normalise=False)
    assert call.ids[:3].cpu().tolist() == [[0, 3]] * 3
    p = np.exp(np.arange(5.)) / np.exp(np.arange(5.)).sum()
    assert np.allclose(call.weights[:3].cpu().numpy(), p[[0, 3]], rtol=1e-6, atol=0)
    assert call.counts.cpu().tolist() == [3, 0, 0, 3, 0, 3]
    # A score is one addition in fp32: 1 and 1 + 2^-30 are one score, and the lower number's.
    small = ebag.MoePerm(1, 1, 3)
    logits = torch.tensor([[0.0, 2.0 ** -30, 2.0 ** -30]], device="cuda")
    call = Call(small, logits, 1, 3, False, bias=torch.ones(3, device="cuda"))
    assert call.ids[0, 0] == 0
    plan.close()
    small.close()


def test_no_tokens():
    import torch
    import paper_2305_06942_amd as ebag
    plan = ebag.MoePerm(4, 2, 7)
    logits = torch.empty((0, 7), device="cuda")
    call = Call(plan, logits, 2, 7, True)
    assert (call.ids == -77).all() and call.counts.eq(0).all() and call.sums.eq(0).all() and call.losses.eq(0).all()
    Call(plan, logits, 2, 7, False)
    plan.choose_backward(logits, call.ids[:0], call.weights[:0], logits)
    plan.close()


def test_captured_and_replayed_with_eager_calls_between():
    """Choice with totals and its gradient in a graph, on another stream than the tensors' own, replayed with new logits."""
    import torch
    import paper_2305_06942_amd as ebag
    rng = np.random.default_rng(73)
    N, k, E = 6000, 4, 96
    plan = ebag.MoePerm(N, k, E)
    logits, eager = torch.empty((N, E), device="cuda"), torch.empty((N, E), device="cuda")
    logits.normal_()
    call = Call(plan, logits, k, E)
    other = Call(plan, eager.normal_(), k, E)
    dw, dl = torch.randn((N, k), device="cuda"), torch.tensor((2.0, 3.0), device="cuda")
    out, out2 = torch.empty_like(logits), torch.empty_like(logits)
    back = lambda c, x, o: plan.choose_backward(x, c.ids[:N], dw, o, counts=c.counts, dlosses=dl)  # noqa: E731
    back(call, logits, out)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            call.again()
            back(call, logits, out)
    for _ in range(4):
        new = torch.from_numpy(rng.standard_normal((N, E)).astype(np.float32)).cuda()
        logits.copy_(new)
        eager.copy_(new)
        call.weights.fill_(float("nan"))
        out.fill_(float("nan"))
        graph.replay()
        other.again()
        back(other, eager, out2)
        torch.cuda.synchronize()
        for x, y in zip(call.outputs(), other.outputs()):
            assert torch.equal(x.nan_to_num(7), y.nan_to_num(7))
        assert torch.equal(out, out2)
    plan.close()


def test_into_the_sort():
    """The choices go into the sort as they are: its offsets are the counts' running sums, without the dropped."""
    import torch
    import paper_2305_06942_amd as ebag
    rng = np.random.default_rng(74)
    N, k, E = 5000, 6, 60
    plan = ebag.MoePerm(N, k, E)
    live = torch.from_numpy(rng.random(N) > 0.3).cuda()
    call = Call(plan, _logits(rng, N, E, "bfloat16", 0.4), k, E, live=live)
    new = lambda *s: torch.empty(s, dtype=torch.int32, device="cuda")  # noqa: E731
    offsets, pos, src = new(E + 1), new(N, k), new(N * k)
    plan.sort(call.ids[:N], offsets, pos, src)
    assert torch.equal(offsets[1:] - offsets[:-1], call.counts[:-1])
    plan.close()

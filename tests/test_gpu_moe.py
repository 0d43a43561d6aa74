"""Tokens by expert (ebag_a2a_moe_*) against the definition in 64 bits.

The order is a matter of whole numbers and compared exactly; so are copies
(dispatch) and single products rounded once (dys).  Sums: a chain of n fp32
fused multiply-adds is off by at most n 2^-24 sum|terms| to first order, so it
lies within b = (n + 1) 2^-24 sum|terms| of the sum in 64 bits; rounding to the
storage type keeps order, so the result lies between want - b and want + b,
both rounded to that type.  A dot product's chain is ceil(V / 64) vectors of N elements on a lane, the elements behind
them, and six levels across the lanes; rows of fewer than 33 vectors have a
lane to a vector."""
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


def _order(ids, E):
    """(offsets, pos, src) by the definition."""
    flat = ids.reshape(-1)
    key = np.where((flat >= 0) & (flat < E), flat, E)
    src = np.argsort(key, kind="stable")
    pos = np.empty(len(flat), dtype=np.int32)
    pos[src] = np.arange(len(flat))
    return np.searchsorted(key[src], np.arange(E + 1)).astype(np.int32), pos.reshape(ids.shape), src.astype(np.int32)


def _ids(rng, N, k, E, dropped):
    ids = rng.integers(0, E, size=(N, k)).astype(np.int32)
    if dropped:
        bad = rng.random((N, k)) < dropped
        ids[bad] = rng.choice([-1, E, E + 7, np.iinfo(np.int32).min, np.iinfo(np.int32).max], size=int(bad.sum()))
    return ids


def _sorted(plan, ids, E):
    import torch
    n = ids.size
    dev = torch.from_numpy(ids).cuda()
    offsets = torch.full((E + 1,), -7, dtype=torch.int32, device="cuda")
    pos = torch.full(ids.shape, -7, dtype=torch.int32, device="cuda")
    src = torch.full((n,), -7, dtype=torch.int32, device="cuda")
    plan.sort(dev, offsets, pos, src)
    return offsets, pos, src


@pytest.mark.parametrize("N,k,E,dropped", [
    (0, 2, 5, 0), (1, 1, 1, 0), (1, 1, 1, 1.0), (1, 8, 512, 0), (5, 3, 7, 0.3), (63, 1, 2, 0), (64, 1, 64, 0),
    (32, 8, 128, 0), (257, 4, 60, 0.1), (1024, 4, 3, 0), (1025, 4, 512, 0.5), (4096, 1, 1, 0), (4097, 1, 511, 0),
    (2731, 6, 100, 0.05), (16384, 1, 256, 0), (16385, 1, 256, 0), (20000, 8, 256, 0.01), (9001, 64, 17, 0.2),
    (70001, 9, 512, 0.001), (3000, 2, 8, 1.0)])
def test_sort(N, k, E, dropped):
    import torch
    import paper_2305_06942_amd as ebag
    rng = np.random.default_rng([41, N, k, E])
    plan = ebag.MoePerm(N, k, E)
    for ids in (_ids(rng, N, k, E, dropped), np.full((N, k), E - 1, dtype=np.int32)):
        got = _sorted(plan, ids, E)
        for g, want, what in zip(got, _order(ids, E), ("offsets", "pos", "src")):
            assert np.array_equal(g.cpu().numpy(), want), what
    plan.close()
    torch.cuda.synchronize()


def _t(a, dtype):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).to(getattr(torch, dtype)).cuda()


def _strided(rows, cols, dtype, step, shift, fill=None):
    """A [rows, cols] view with `step` elements between rows, `shift` elements
    behind its allocation's start; and the allocation, filled with NaN."""
    import torch
    buf = torch.full((rows * step + shift + 16,), float("nan"), dtype=getattr(torch, dtype), device="cuda")
    view = buf[shift:shift + rows * step].view(rows, step)[:, :cols]
    if fill is not None:
        view.copy_(fill)
    return view, buf


def _f64(t):
    return t.detach().double().cpu().numpy()


def _close(got, want, terms, chain, dtype):
    import torch
    b = (chain + 1) * 2.0 ** -24 * terms
    lo, hi = (torch.from_numpy(v).to(getattr(torch, dtype)).double().numpy() for v in (want - b, want + b))
    ok = (lo <= got) & (got <= hi)
    assert np.all(ok), f"{got[~ok][0]} outside [{lo[~ok][0]}, {hi[~ok][0]}], {int((~ok).sum())} in all"


def _chain(dim, dtype):
    n = 4 if dtype == "float32" else 8
    vecs = dim // n
    return -(-vecs // 64) * n + n + 7


SHAPES = [  # tokens, choices, experts, dim, step, shift, dropped
    (1, 1, 1, 1, 1, 0, 0), (1, 2, 4, 3, 5, 1, 0), (3, 2, 4, 7, 7, 0, 0.5), (5, 3, 2, 8, 8, 0, 0),
    (17, 4, 8, 33, 40, 3, 0.2), (40, 8, 16, 64, 64, 0, 0), (33, 5, 8, 250, 250, 1, 0.1), (64, 8, 128, 256, 264, 0, 0),
    (12, 9, 30, 519, 520, 0, 0.1), (7, 2, 3, 1999, 1999, 0, 0.3), (9, 17, 40, 1024, 1024, 0, 0.1),
    (130, 2, 8, 4096, 4096, 0, 0), (6, 4, 5, 9000, 9001, 5, 0.2), (11, 3, 4, 130, 130, 0, 1.0)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,k,E,D,step,shift,dropped", SHAPES)
def test_rows(N, k, E, D, step, shift, dropped, dtype):
    """All four row operators; dropped rows of the inputs hold NaN, and nothing
    between or behind the outputs' rows is written."""
    import torch
    import paper_2305_06942_amd as ebag
    rng = np.random.default_rng([42, N, k, D, TYPES.index(dtype)])
    plan = ebag.MoePerm(N, k, E)
    ids = _ids(rng, N, k, E, dropped)
    offsets, pos, _ = _sorted(plan, ids, E)
    off, p, _ = _order(ids, E)
    S, kept = N * k, p < off[E]
    flat, flat_kept = p.reshape(-1), kept.reshape(-1)

    def rows(n, poison=False):
        v = rng.standard_normal((n, D))
        if poison:
            v[off[E]:] = np.nan
        return _strided(n, D, dtype, step, shift, _t(v, dtype))[0]

    def result(n):
        return _strided(n, D, dtype, step, shift)

    def untouched(buf, n):
        used = torch.zeros(buf.numel(), dtype=torch.bool, device="cuda")
        used[shift:shift + n * step].view(n, step)[:, :D] = True
        assert torch.isnan(buf[~used]).all(), "written outside the rows"

    w = rng.standard_normal((N, k)).astype(np.float32)
    w[~kept] = np.nan  # a dropped choice's weight is not used either
    dw_dev = torch.full((N, k), float("nan"), device="cuda")
    w_dev = torch.from_numpy(w).cuda()
    w64 = np.where(kept, w, 0).astype(np.float64)

    x = rows(N)
    xs, buf = result(S)
    plan.dispatch(x, offsets, pos, xs)
    want = np.zeros((S, D))
    want[flat[flat_kept]] = np.repeat(_f64(x), k, axis=0)[flat_kept]
    assert np.array_equal(_f64(xs), want)
    untouched(buf, S)

    dxs = rows(S, True)
    dx, buf = result(N)
    plan.dispatch_backward(dxs, offsets, pos, dx)
    picked = np.where(kept[..., None], _f64(dxs)[p], 0)
    _close(_f64(dx), picked.sum(1), np.abs(picked).sum(1), k, dtype)
    untouched(buf, N)

    ys = rows(S, True)
    out, buf = result(N)
    plan.combine(ys, offsets, pos, w_dev, out)
    picked = np.where(kept[..., None], _f64(ys)[p], 0)
    terms = picked * w64[..., None]
    _close(_f64(out), terms.sum(1), np.abs(terms).sum(1), k, dtype)
    untouched(buf, N)

    dout = rows(N)
    dys, buf = result(S)
    plan.combine_backward(dout, ys, offsets, pos, w_dev, dys, dw_dev)
    scaled = (w_dev.nan_to_num()[..., None] * dout.float()[:, None, :]).to(dys.dtype)  # one product, rounded once
    scaled = np.where(kept[..., None], _f64(scaled), 0).reshape(S, D)
    want = np.zeros((S, D))
    want[flat] = scaled
    assert np.array_equal(_f64(dys), want)
    untouched(buf, S)
    terms = picked * _f64(dout)[:, None, :]
    _close(_f64(dw_dev), terms.sum(2), np.abs(terms).sum(2), _chain(D, dtype), "float32")
    plan.close()


def test_gradients_match_differences():
    """combine and dispatch are linear in each input: with whole numbers small
    enough for fp32, a step's difference is the derivative, bit for bit."""
    import torch
    import paper_2305_06942_amd as ebag
    N, k, E, D = 6, 3, 4, 37
    rng = np.random.default_rng(43)
    plan = ebag.MoePerm(N, k, E)
    offsets, pos, _ = _sorted(plan, _ids(rng, N, k, E, 0.2), E)
    whole = lambda *s: torch.from_numpy(rng.integers(-9, 10, size=s).astype(np.float32)).cuda()  # noqa: E731
    ys, w, dout, x, dxs = whole(N * k, D), whole(N, k), whole(N, D), whole(N, D), whole(N * k, D)
    dys, dw, dx = torch.empty_like(ys), torch.empty_like(w), torch.empty_like(x)
    plan.combine_backward(dout, ys, offsets, pos, w, dys, dw)
    plan.dispatch_backward(dxs, offsets, pos, dx)

    def loss(ys, w):
        out = torch.empty_like(dout)
        plan.combine(ys, offsets, pos, w, out)
        return float((out.double() * dout.double()).sum())

    def loss_x(x):
        xs = torch.empty_like(dxs)
        plan.dispatch(x, offsets, pos, xs)
        return float((xs.double() * dxs.double()).sum())

    base, base_x = loss(ys, w), loss_x(x)
    for n in range(N):
        for j in range(k):
            v = w.clone()
            v[n, j] += 1
            assert loss(ys, v) - base == float(dw[n, j])
    for r, c in [(r, c) for r in range(N * k) for c in (0, 5, 31, 36)]:
        v = ys.clone()
        v[r, c] += 1
        assert loss(v, w) - base == float(dys[r, c])
    for n, c in [(n, c) for n in range(N) for c in (0, 3, 32, 36)]:
        v = x.clone()
        v[n, c] += 1
        assert loss_x(v) - base_x == float(dx[n, c])
    plan.close()


def test_infinite_and_nan_rows_stay_their_own():
    """A kept row's infinities and NaN reach its own token only."""
    import torch
    import paper_2305_06942_amd as ebag
    N, k, E, D = 10, 2, 3, 100
    rng = np.random.default_rng(44)
    plan = ebag.MoePerm(N, k, E)
    offsets, pos, src = _sorted(plan, _ids(rng, N, k, E, 0), E)
    ys = torch.ones((N * k, D), device="cuda")
    ys[pos[3, 1].long(), 7] = float("inf")
    ys[pos[5, 0].long(), 99] = float("nan")
    w = torch.full((N, k), 0.5, device="cuda")
    out = torch.empty((N, D), device="cuda")
    plan.combine(ys, offsets, pos, w, out)
    want = torch.ones((N, D), device="cuda")
    want[3, 7], want[5, 99] = float("inf"), float("nan")
    assert torch.equal(out.nan_to_num(nan=-3.0), want.nan_to_num(nan=-3.0))
    plan.close()


def test_foreign_places_stay_in_range():
    """Places that no sort made are treated as dropped where they lie outside
    the rows; an offset above the rows counts as all of them."""
    import torch
    import paper_2305_06942_amd as ebag
    N, k, E, D = 4, 2, 2, 64
    plan = ebag.MoePerm(N, k, E)
    offsets = torch.tensor([0, 4, 1 << 30], dtype=torch.int32, device="cuda")
    pos = torch.tensor([[0, 1], [2, 3], [-1, 8], [1 << 30, 5]], dtype=torch.int32, device="cuda")
    ys = torch.ones((N * k, D), device="cuda")
    w = torch.ones((N, k), device="cuda")
    out = torch.empty((N, D), device="cuda")
    plan.combine(ys, offsets, pos, w, out)
    assert out[:, 0].tolist() == [2, 2, 0, 1]
    dys, dw = torch.full_like(ys, 5), torch.empty_like(w)
    plan.combine_backward(torch.ones((N, D), device="cuda"), ys, offsets, pos, w, dys, dw)
    assert dw.tolist() == [[D, D], [D, D], [0, 0], [0, D]]
    assert dys[:, 0].tolist() == [1, 1, 1, 1, 5, 1, 5, 5]
    plan.close()


def test_second_stream_is_refused_while_a_large_sort_runs_and_graph_replays_match():
    import torch
    import paper_2305_06942_amd as ebag
    N, k, E = 60000, 8, 256
    rng = np.random.default_rng(45)
    plan = ebag.MoePerm(N, k, E)
    ids = torch.empty((N, k), dtype=torch.int32, device="cuda")
    offsets = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    pos, src = torch.zeros_like(ids), torch.zeros(N * k, dtype=torch.int32, device="cuda")
    x = torch.randn((N, 8), device="cuda")
    xs = torch.zeros((N * k, 8), device="cuda")
    side = torch.cuda.Stream()
    ids.copy_(torch.from_numpy(_ids(rng, N, k, E, 0)))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan.sort(ids, offsets, pos, src)
        plan.dispatch(x, offsets, pos, xs)
    for _ in range(4):
        new = _ids(rng, N, k, E, 0.02)
        ids.copy_(torch.from_numpy(new))
        x.normal_()
        graph.replay()
        torch.cuda.synchronize()
        off, p, s = _order(new, E)
        assert np.array_equal(offsets.cpu().numpy(), off) and np.array_equal(pos.cpu().numpy(), p)
        assert np.array_equal(src.cpu().numpy(), s)
        want = torch.zeros_like(xs)
        want[:off[E]] = x[src[:off[E]].long() // k]
        assert torch.equal(xs, want)
    # Work ahead of the sort keeps it from completing while the second is asked for.
    a = torch.randn((8192, 8192), device="cuda")
    for _ in range(4):
        a = a @ a * 1e-4
    plan.sort(ids, offsets, pos, src)
    with pytest.raises(ebag.EbagError, match="sort of this plan is still running"):
        plan.sort(ids, offsets, pos, src, stream=side)
    torch.cuda.synchronize()
    plan.sort(ids, offsets, pos, src, stream=side)
    side.synchronize()
    assert np.array_equal(offsets.cpu().numpy(), off) and np.array_equal(src.cpu().numpy(), s)
    plan.close()


def test_rows_on_a_stream_of_their_own():
    """Calls run on the stream they are given: behind work that is still in it."""
    import torch
    import paper_2305_06942_amd as ebag
    N, k, E, D = 500, 2, 8, 512
    rng = np.random.default_rng(46)
    plan = ebag.MoePerm(N, k, E)
    offsets, pos, _ = _sorted(plan, _ids(rng, N, k, E, 0), E)
    side = torch.cuda.Stream()
    x = torch.zeros((N, D), device="cuda")
    xs, back = torch.zeros((N * k, D), device="cuda"), torch.zeros((N, D), device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        a = torch.randn((4096, 4096), device="cuda")
        for _ in range(8):
            a = a @ a * 1e-4
        x.fill_(3.0)
        plan.dispatch(x, offsets, pos, xs)
        plan.dispatch_backward(xs, offsets, pos, back)
    side.synchronize()
    assert bool((back == 6.0).all())
    plan.close()


@pytest.mark.parametrize("N,k,D,dtype", [(9000, 8, 1024, "bfloat16"), (11000, 6, 1021, "float16"), (70000, 8, 64, "float32")])
def test_rows_that_go_past_the_caches(N, k, D, dtype):
    """Rows by place of more than 128 MiB, whole cache lines and not, in whole
    numbers: sums of products below 2^24 leave fp32 nothing to round, so each
    result is the exact one rounded once."""
    import torch
    import paper_2305_06942_amd as ebag
    E = 40
    assert N * k * D * (4 if dtype == "float32" else 2) > 128 << 20
    g = torch.Generator(device="cuda").manual_seed(47)
    t = getattr(torch, dtype)
    whole = lambda *s: torch.randint(-9, 10, s, generator=g, device="cuda").to(t)  # noqa: E731
    plan = ebag.MoePerm(N, k, E)
    ids = torch.randint(-1, E, (N, k), generator=g, device="cuda", dtype=torch.int32)
    offsets = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    pos, src = torch.zeros_like(ids), torch.zeros(N * k, dtype=torch.int32, device="cuda")
    plan.sort(ids, offsets, pos, src)
    total = int(offsets[-1])
    kept = (pos < total)[..., None]
    assert 0 < total < N * k
    x, w = whole(N, D), torch.randint(-9, 10, (N, k), generator=g, device="cuda").float()
    xs, out = torch.full((N * k, D), float("nan"), dtype=t, device="cuda"), torch.full((N, D), float("nan"), dtype=t, device="cuda")
    plan.dispatch(x, offsets, pos, xs)
    want = torch.where(torch.arange(N * k, device="cuda")[:, None] < total, x[src.long() // k], 0)
    assert torch.equal(xs, want)
    ys = whole(N * k, D)
    ys[total:] = float("nan")
    rows = torch.where(kept, ys[pos.long()].float(), 0)
    plan.combine(ys, offsets, pos, w, out)
    assert torch.equal(out, (rows * w[..., None]).sum(1).to(t))
    plan.dispatch_backward(ys, offsets, pos, out)
    assert torch.equal(out, rows.sum(1).to(t))
    dys, dw = torch.full_like(xs, float("nan")), torch.full_like(w, float("nan"))
    plan.combine_backward(x, ys, offsets, pos, w, dys, dw)
    assert torch.equal(dw, (rows * x.float()[:, None]).sum(2))
    want = torch.zeros_like(dys)
    want[pos.long().reshape(-1)] = torch.where(kept, w[..., None] * x.float()[:, None], 0).to(t).reshape(N * k, D)
    assert torch.equal(dys, want)
    plan.close()

"""Products in 8-bit integers (gemv_ar_q8_*) against the definition in 64 bits.

Codes, scales and sums are exact: codes are compared as they are, and with u =
2^-24 a result is off by one rounding each of the sum to fp32, of the two scales'
product and of the whole: 3 u and a little, 4 u |y|.  silu(g) = g / (1 + exp(-g)) with
an exponential good to (|g| + 8) 2^-22 and a slope of at most 1.1 carries that on.
Rounding to the storage type keeps order, so a result lies between want - b and
want + b, both rounded."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

TYPES = ("float32", "float16", "bfloat16")
U = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    torch.cuda.set_device(0)
    yield
    torch.cuda.synchronize()


def _plan(M, K, dtype, experts=1, glu=0):
    import paper_2305_06942_amd as ebag
    return ebag.Q8Gemv(M, K, TYPES.index(dtype), experts=experts, glu=glu)


def _strided(rows, cols, dtype, step, shift, values=None):
    """A [rows, cols] view with cols + step elements between rows, `shift` behind its allocation's start, which holds NaN."""
    import torch
    buf = torch.full((rows * (cols + step) + shift + 32,), float("nan"), dtype=getattr(torch, dtype), device="cuda")
    view = buf[shift:shift + rows * (cols + step)].view(rows, cols + step)[:, :cols]
    if values is not None:
        view.copy_(torch.from_numpy(values).to(getattr(torch, dtype)))
    return view, buf


def _untouched(buf, rows, cols, step, shift):
    import torch
    outside = torch.ones_like(buf, dtype=torch.bool)
    outside[shift:shift + rows * (cols + step)].view(rows, cols + step)[:, :cols] = False
    assert buf[outside].isnan().all(), "written outside the rows"


def _rounded(x64):
    """(codes, scales) of rows by the definition, in 64 bits."""
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        top = np.abs(x64).max(1)
        fine = np.isfinite(x64).all(1)
        scale = (top / 127).astype(np.float32)
        q = np.rint(x64 / scale.astype(np.float64)[:, None])
        codes = np.where((fine & (scale > 0))[:, None], np.clip(q, -127, 127), 0.0)
    return codes, np.where(fine, scale, np.nan).astype(np.float32)


def _scratch(plan, rows):
    """xq and xs that hold something else."""
    import torch
    return (torch.full((rows, plan.pitch), 99, dtype=torch.int8, device="cuda"), torch.full((rows,), 3.25, device="cuda"))


class Weights:
    def __init__(self, rng, plan, M, K, E=1, lowest=-128):
        import torch
        self.c64 = rng.integers(lowest, 128, size=(E, M, K)).astype(np.float64)
        codes = rng.integers(-128, 128, size=(E, M, plan.pitch)).astype(np.int8)  # any numbers behind column K
        codes[..., :K] = self.c64
        self.codes = torch.from_numpy(codes).cuda()
        self.scales = torch.from_numpy((rng.uniform(0.5, 1.5, size=(E, M)) / (73 * np.sqrt(K))).astype(np.float32)).cuda()
        self.s64 = self.scales.double().cpu().numpy()


def _want(xq64, xs64, w, e, glu):
    """(result, its bound)."""
    y = (xq64 @ w.c64[e].T) * xs64[:, None] * w.s64[e][None]
    b = 4 * U * np.abs(y) + 2.0 ** -149
    if not glu:
        return y, b
    half = y.shape[1] // 2
    g, u, bg, bu = y[:, :half], y[:, half:], b[:, :half], b[:, half:]
    act = g / (1 + np.exp(-g))
    ba = 1.1 * bg + (np.abs(g) + 8) * 2.0 ** -22 * np.abs(act)
    return act * u, ba * np.abs(u) + np.abs(act) * bu + ba * bu + U * np.abs(act * u)


def _check(got, want, b, y_dtype, what=""):
    import torch
    got = got.double().cpu().numpy()
    lo, hi = (torch.from_numpy(v).to(getattr(torch, y_dtype)).double().numpy() for v in (want - b, want + b))
    ok = (lo <= got) & (got <= hi)
    assert np.all(ok), f"{what}{int((~ok).sum())} of {ok.size} outside, the first at {np.argwhere(~ok)[0]}: {got[~ok][0]} not in [{lo[~ok][0]}, {hi[~ok][0]}]"


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,K,step,shift", [
    (1, 1, 0, 0), (1, 7, 0, 1), (3, 8, 3, 0), (5, 127, 1, 3), (4, 128, 0, 0), (9, 129, 0, 5), (6, 1000, 24, 0), (7, 2048, 0, 0), (3, 2049, 0, 1),
    (2, 5001, 7, 2), (5, 8192, 0, 0), (3, 8200, 0, 0), (2, 20003, 0, 1), (1, 131072, 0, 0), (1000, 64, 0, 0), (4099, 40, 0, 0)])
def test_round(rows, K, step, shift, dtype):
    import torch
    rng = np.random.default_rng([81, rows, K])
    plan = _plan(4, K, dtype)
    x, _ = _strided(rows, K, dtype, step, shift, rng.standard_normal((rows, K)) * 10.0 ** rng.integers(-4, 5, size=(rows, 1)) * 0.5)
    if rows > 2:
        x[1] = 0
    xq, xs = _scratch(plan, rows)
    plan.round(x, xq, xs)
    codes, scales = _rounded(x.double().cpu().numpy())
    assert np.array_equal(xs.cpu().numpy(), scales), "scales"
    got = xq.cpu().numpy()
    assert np.array_equal(got[:, :K], codes), "codes"
    assert not got[:, K:].any(), "behind the row's end"
    if dtype != "float32" or rows < 1000:
        w = torch.empty((1, 4, K), dtype=x.dtype, device="cuda").normal_()
        wq, ws = torch.empty((1, 4, plan.pitch), dtype=torch.int8, device="cuda"), torch.empty((1, 4), device="cuda")
        plan.quantize(w, wq, ws)
        codes, scales = _rounded(w[0].double().cpu().numpy())
        assert np.array_equal(wq[0, :, :K].cpu().numpy(), codes) and np.array_equal(ws[0].cpu().numpy(), scales)
    plan.close()


def test_round_ties_and_neighbours():
    """Numbers in the middle of two codes and next to it: the largest is 127 times a power of two, so that scales are
    exact, from the smallest numbers of fp32 to the largest."""
    import torch
    plan = _plan(4, 509, "float32")
    rows = []
    for power in (-149, -148, -140, -127, -126, -100, -70, -61, -60, -59, -30, 0, 5, 100, 120):
        mid = (np.arange(-127, 127) + 0.5) * 2.0 ** power
        with np.errstate(under="ignore"):
            mid = mid.astype(np.float32)
            row = np.concatenate(([127 * 2.0 ** power], mid, np.nextafter(mid, np.float32(np.inf)), np.zeros(0))).astype(np.float32)
            rows += [row, np.concatenate((row[:255], np.nextafter(mid, -np.float32(np.inf)))).astype(np.float32)]
    rows += [np.full(509, v, dtype=np.float32) for v in (1e-45, -9e-44, 1.2e-43, 2.6e-43, 3.4028235e38, 1.1754944e-38)]
    rows += [np.float32(2.0) ** np.linspace(-149, 127, 509).astype(np.float32)]
    x = np.stack(rows)
    xq, xs = _scratch(plan, len(rows))
    plan.round(torch.from_numpy(x).cuda(), xq, xs)
    codes, scales = _rounded(x.astype(np.float64))
    assert np.array_equal(xs.cpu().numpy(), scales)
    bad = np.argwhere(xq.cpu().numpy()[:, :509] != codes)
    assert not len(bad), (bad[0], x[tuple(bad[0])], codes[tuple(bad[0])], xq.cpu().numpy()[tuple(bad[0])])
    plan.close()


@pytest.mark.parametrize("dtype,bits", [("float16", "int16"), ("bfloat16", "int16")])
def test_round_every_bit_pattern(dtype, bits):
    """Every finite 16-bit number in rows of its own sign and exponent's neighbourhood."""
    import torch
    K = 256
    plan = _plan(4, K, dtype)
    x = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(getattr(torch, dtype)).view(256, K)
    x = torch.where(torch.isfinite(x), x, torch.ones_like(x)).cuda()
    xq, xs = _scratch(plan, 256)
    plan.round(x, xq, xs)
    codes, scales = _rounded(x.double().cpu().numpy())
    assert np.array_equal(xs.cpu().numpy(), scales) and np.array_equal(xq.cpu().numpy(), codes)
    plan.close()


FORWARD = [  # rows, M, K, glu, step, shift
    (1, 1, 1, 0, 0, 0), (1, 2, 3, 1, 1, 1), (1, 16, 128, 0, 0, 0), (2, 17, 129, 0, 3, 1), (4, 64, 1000, 1, 0, 0), (1, 513, 4096, 0, 0, 0),
    (12, 301, 5001, 0, 1, 3), (16, 34, 640, 1, 0, 0), (17, 100, 256, 0, 0, 0), (31, 70, 384, 1, 5, 1), (33, 48, 2100, 0, 0, 0), (64, 130, 300, 1, 0, 0),
    (1, 70000, 200, 0, 0, 0), (3, 66000, 130, 1, 0, 0), (64, 5000, 130, 0, 0, 0),
    # Few rows: one row and two on 16-byte boundaries (rounded by the product) and off them, in both types of tiles; waves that
    # share x by 2, 4 and 8; two, three and more tiles of x that share weights.
    (1, 4096, 1024, 0, 0, 0), (2, 300, 512, 1, 8, 8), (2, 7000, 136, 0, 16, 0), (2, 300, 512, 1, 4, 0), (1, 13000, 64, 1, 0, 0), (2, 48, 12288, 0, 0, 0),
    (16, 13001, 140, 0, 0, 0), (32, 13000, 130, 0, 0, 1), (32, 26000, 130, 1, 0, 0), (20, 3300, 2000, 0, 0, 0), (64, 26001, 140, 0, 1, 0),
    (64, 52000, 130, 1, 0, 0), (50, 7000, 140, 0, 0, 0), (40, 500, 3000, 1, 0, 0), (96, 2000, 520, 0, 0, 0), (150, 400, 700, 1, 0, 0),
    (65, 5, 100, 0, 0, 0), (65, 256, 128, 0, 0, 0), (100, 258, 1000, 1, 2, 1), (129, 300, 513, 0, 0, 0), (200, 1030, 260, 1, 0, 0),
    (257, 255, 129, 0, 1, 1), (700, 514, 384, 1, 0, 0), (1025, 700, 640, 0, 0, 0), (1300, 1400, 200, 1, 0, 3), (3000, 40, 128, 0, 0, 0),
    (2000, 6200, 129, 0, 0, 0), (6100, 2050, 300, 1, 1, 1), (4100, 4104, 257, 0, 0, 0), (1500, 2100, 1100, 0, 0, 0)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,M,K,glu,step,shift", FORWARD)
def test_forward(rows, M, K, glu, step, shift, dtype):
    import torch
    rng = np.random.default_rng([82, rows, M, K])
    plan = _plan(M, K, dtype, glu=glu)
    w = Weights(rng, plan, M, K)
    x, _ = _strided(rows, K, dtype, step, shift, rng.standard_normal((rows, K)))
    xq64, xs64 = _rounded(x.double().cpu().numpy())
    want, b = _want(xq64, xs64.astype(np.float64), w, 0, glu)
    xq, xs = _scratch(plan, rows)
    for y_dtype in {dtype, "float32"}:
        y, buf = _strided(rows, plan.wide, y_dtype, step, shift)
        plan.forward(w.codes, w.scales, x, y, xq, xs)
        _check(y, want, b, y_dtype)
        _untouched(buf, rows, plan.wide, step, shift)
    plan.round(x, xq, xs)  # and from rows that are rounded already
    again = torch.full_like(y, float("nan"))
    plan.forward(w.codes, w.scales, None, again, xq, xs)
    assert torch.equal(again, y)
    plan.close()


@pytest.mark.parametrize("rows", [1, 3, 20, 70, 300])
def test_largest_sums(rows):
    """Sums next to the ends of 32 bits: 127 * 128 * 2^17 with every sign."""
    import torch
    K, M = 1 << 17, 6
    plan = _plan(M, K, "float32")
    codes = torch.tensor([127, -128, 1, -1, 0, 127], dtype=torch.int8, device="cuda").view(1, M, 1).expand(1, M, K).contiguous()
    scales = torch.ones((1, M), device="cuda")
    sign = torch.ones(rows, 1, device="cuda")
    sign[1::2] = -1
    x = (sign * 127).expand(rows, K).contiguous()
    xq, xs = _scratch(plan, rows)
    y = torch.empty((rows, M), device="cuda")
    plan.forward(codes, scales, x, y, xq, xs)
    want = (sign.double() * 127 * K * codes[0, :, 0].double()).float()
    assert torch.equal(y, want)
    plan.close()


def _offsets(rng, rows, E, dropped, empty):
    """Rows of each expert, some without any, the last `dropped` of nobody."""
    p = rng.random(E) ** 2 + 1e-3
    p[rng.random(E) < empty] = 0
    if not p.any():
        p[0] = 1
    counts = rng.multinomial(rows - dropped, p / p.sum())
    return np.concatenate(([0], np.cumsum(counts))).astype(np.int32)


EXPERTS = [  # rows, E, M, K, glu, k, dropped, empty
    (1, 1, 16, 128, 0, 1, 0, 0), (1, 9, 5, 100, 0, 1, 1, 0), (8, 70, 34, 129, 1, 2, 1, 0.5), (64, 130, 20, 256, 0, 4, 5, 0.3), (300, 60, 70, 250, 1, 3, 17, 0),
    (256, 8, 130, 384, 0, 8, 0, 0.3), (500, 8, 66, 130, 1, 4, 33, 0), (900, 9, 300, 200, 0, 3, 100, 0.2), (2000, 12, 514, 128, 1, 8, 0, 0),
    (2600, 2, 260, 256, 0, 2, 7, 0), (1200, 512, 8, 64, 0, 1, 3, 0.5), (6000, 4, 130, 130, 1, 6, 1000, 0.3),
    (40, 3, 3000, 260, 0, 2, 0, 0), (70, 40, 700, 300, 1, 2, 2, 0.2), (5000, 6, 2100, 260, 1, 4, 50, 0.2), (400, 3, 4100, 130, 0, 1, 0, 0)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,E,M,K,glu,k,dropped,empty", EXPERTS)
def test_experts(rows, E, M, K, glu, k, dropped, empty, dtype):
    import torch
    rng = np.random.default_rng([83, rows, E, M, K])
    plan = _plan(M, K, dtype, experts=E, glu=glu)
    w = Weights(rng, plan, M, K, E)
    ends = _offsets(rng, rows, E, dropped, empty)
    offsets = torch.from_numpy(ends).cuda()
    tokens = -(-rows // k)
    src = rng.permutation(tokens * k)[:rows].astype(np.int32)
    for gather in (False, True):
        n = tokens if gather else rows
        x, _ = _strided(n, K, dtype, 5, 1, rng.standard_normal((n, K)))
        xq64, xs64 = _rounded(x.double().cpu().numpy())
        if gather:
            xq64, xs64 = xq64[src // k], xs64[src // k]
        want, b = np.zeros((rows, plan.wide)), np.zeros((rows, plan.wide))
        for e in range(E):
            at = slice(ends[e], ends[e + 1])
            if ends[e + 1] > ends[e]:
                want[at], b[at] = _want(xq64[at], xs64[at].astype(np.float64), w, e, glu)
        xq, xs = _scratch(plan, n)
        y, buf = _strided(rows, plan.wide, dtype, 3, 1)
        plan.experts(w.codes, w.scales, x, offsets, y, xq, xs, src=torch.from_numpy(src).cuda() if gather else None, k=k)
        _check(y, want, b, dtype, f"gather {gather}: ")
        _untouched(buf, rows, plan.wide, 3, 1)
    plan.close()


@pytest.mark.parametrize("rows,glu", [(5, 0), (5, 1), (40, 0), (300, 1), (1100, 0)])
def test_rows_that_are_not_numbers(rows, glu):
    """An infinity or NaN makes its own row NaN and no other; a row of zeros gives zeros."""
    import torch
    rng = np.random.default_rng(84)
    M, K = 70, 300
    plan = _plan(M, K, "bfloat16", glu=glu)
    w = Weights(rng, plan, M, K)
    x = torch.from_numpy(rng.standard_normal((rows, K))).to(torch.bfloat16).cuda()
    clean = torch.empty((rows, plan.wide), device="cuda")
    xq, xs = _scratch(plan, rows)
    plan.forward(w.codes, w.scales, x, clean, xq, xs)
    x[0, 7], x[2, 299], x[4], x[3] = float("nan"), -float("inf"), float("inf"), 0
    y = torch.empty_like(clean)
    plan.forward(w.codes, w.scales, x, y, xq, xs)
    bad = [0, 2, 4]
    assert y[bad].isnan().all() and xs[bad].isnan().all() and not xq[bad].any()
    assert y[3].eq(0).all() and xs[3] == 0
    rest = [n for n in range(rows) if n not in (0, 2, 3, 4)]
    assert torch.equal(y[rest], clean[rest])
    plan.close()


def test_experts_with_offsets_out_of_range_stay_inside():
    """Offsets and src out of range are clamped; what they give is not looked at, only that nothing else is written."""
    import torch
    plan = _plan(40, 130, "float16", experts=3)
    w = Weights(np.random.default_rng(85), plan, 40, 130, 3)
    x = torch.zeros((10, 130), dtype=torch.float16, device="cuda")
    xq, xs = _scratch(plan, 10)
    for bad in ([0, -5, 70, 2 ** 31 - 1], [9, 3, 1, 0], [0, 4, 4, 100]):
        y, buf = _strided(20, 40, "float16", 3, 1)
        plan.experts(w.codes, w.scales, x, torch.tensor(bad, dtype=torch.int32, device="cuda"), y, xq, xs,
                     src=torch.tensor([-1, 2 ** 31 - 1, 500, 19] * 5, dtype=torch.int32, device="cuda"), k=2)
        _untouched(buf, 20, 40, 3, 1)
    plan.close()


def test_no_rows():
    import torch
    plan = _plan(8, 64, "float32")
    w = Weights(np.random.default_rng(86), plan, 8, 64)
    xq, xs = _scratch(plan, 0)
    empty = torch.empty((0, 64), device="cuda")
    plan.round(empty, xq, xs)
    plan.forward(w.codes, w.scales, empty, torch.empty((0, 8), device="cuda"), xq, xs)
    plan.experts(w.codes, w.scales, empty, torch.zeros(2, dtype=torch.int32, device="cuda"), torch.empty((0, 8), device="cuda"), xq, xs)
    plan.close()


@pytest.mark.parametrize("rows", [3, 30, 400])
def test_captured_on_another_stream_and_replayed(rows):
    """Two graphs with scratch of their own and eager calls between, every replay against the eager result."""
    import torch
    rng = np.random.default_rng([87, rows])
    M, K = 300, 700
    plan = _plan(M, K, "bfloat16")
    w = Weights(rng, plan, M, K)
    xs_in = [torch.empty((rows, K), dtype=torch.bfloat16, device="cuda").normal_() for _ in range(3)]
    ys = [torch.empty((rows, M), dtype=torch.bfloat16, device="cuda") for _ in range(3)]
    scratch = [_scratch(plan, rows) for _ in range(3)]
    for i in range(3):
        plan.forward(w.codes, w.scales, xs_in[i], ys[i], *scratch[i])
    side = torch.cuda.Stream()
    graphs = []
    for i in range(2):
        side.wait_stream(torch.cuda.current_stream())
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.stream(side), torch.cuda.graph(graphs[i], stream=side):
            plan.forward(w.codes, w.scales, xs_in[i], ys[i], *scratch[i])
    for _ in range(4):
        for i in range(2):
            xs_in[i].copy_(torch.from_numpy(rng.standard_normal((rows, K))))
            ys[i].fill_(float("nan"))
        graphs[0].replay()
        graphs[1].replay()
        torch.cuda.synchronize()
        for i in range(2):
            plan.forward(w.codes, w.scales, xs_in[i], ys[2], *scratch[2])
            assert torch.equal(ys[2], ys[i])
    plan.close()

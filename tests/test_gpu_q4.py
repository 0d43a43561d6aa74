"""Products with 4-bit weights (gemv_ar_q4_*) against the definition in 64 bits.

Exact inputs: whole x below 2^7, scales that are powers of two and sums below
2^24 leave fp32 nothing to round, so such results are compared bit for bit.

Others: let every term of a sum be at most 62 s |x| and the longest chain 128
products of a group, a multiply-add pair per 32 columns and at most 16 partial
sums; with 2^-23 for each (sums of a matrix instruction need not be rounded to
nearest), |sum - want| <= b = (128 + K / 16 + 16) 2^-23 * 62 sum_k s |x|.  With
fp32 x the terms are (q - zero) s x, at most 15 s |x|.  With fp16 and bf16 x a
code goes as 64 + q or 128 + q, whose part comes off again: terms of up to 286 s
|x|, but a matrix instruction adds 32 columns, 512 columns are 16 steps, and 16 *
286 < 128 * 62.

silu(g) = g / (1 + exp(-g)) with an exponential good to (|g| + 8) 2^-22 and a
slope of at most 1.1 carries b on.  Rounding to the storage type keeps order, so
a result lies between want - b and want + b, both rounded."""
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


def _abi(dtype):
    return TYPES.index(dtype)


class Weights:
    """4-bit weights on the GPU, `at` bytes behind an allocation's start, and their values in 64 bits."""

    def __init__(self, rng, E, M, K, group, dtype, zeros, exact=False, at=3):
        import torch
        rb, groups = (K + 1) // 2, -(-K // group)
        codes = rng.integers(0, 256, size=(E, M, rb), dtype=np.uint8)
        if exact:
            scales = 2.0 ** rng.integers(-3, 2, size=(E, M, groups))
        else:
            scales = rng.uniform(0.5, 1.5, size=(E, M, groups)) / (4.6 * np.sqrt(K))
        z = rng.integers(0, 16, size=(E, M, groups), dtype=np.uint8) if zeros else None
        buf = torch.zeros(codes.size + at, dtype=torch.uint8, device="cuda")
        self.codes = buf[at:].view(E, M, rb)
        self.codes.copy_(torch.from_numpy(codes))
        self.scales = torch.from_numpy(scales).to(getattr(torch, dtype)).cuda()
        self.zeros = None if z is None else torch.from_numpy(z).cuda()
        q = np.empty((E, M, 2 * rb))
        q[..., 0::2], q[..., 1::2] = codes & 15, codes >> 4
        col = np.arange(K) // group
        self.s64 = self.scales.double().cpu().numpy()[..., col]
        self.w64 = self.s64 * (q[..., :K] - (z[..., col] if zeros else 8.0))


def _strided(rows, cols, dtype, step, shift, values=None):
    import torch
    buf = torch.full((rows * step + shift + 32,), float("nan"), dtype=getattr(torch, dtype), device="cuda")
    view = buf[shift:shift + rows * step].view(rows, step)[:, :cols]
    if values is not None:
        view.copy_(torch.from_numpy(values).to(getattr(torch, dtype)))
    return view, buf


def _x(rng, rows, K, dtype, exact, step, shift):
    v = rng.integers(-9, 10, size=(rows, K)).astype(np.float64) if exact else rng.standard_normal((rows, K))
    return _strided(rows, K, dtype, step, shift, v)[0]


def _want(x64, w, e, glu):
    """(result, its bound) of rows x64 on matrix e, in 64 bits."""
    y = x64 @ w.w64[e].T
    b = (144 + x64.shape[1] / 16) * 2.0 ** -23 * 62 * (np.abs(x64) @ w.s64[e].T)
    if not glu:
        return y, b
    half = y.shape[1] // 2
    g, u, bg, bu = y[:, :half], y[:, half:], b[:, :half], b[:, half:]
    act = g / (1 + np.exp(-g))
    ba = 1.1 * bg + (np.abs(g) + 8) * 2.0 ** -22 * np.abs(act)
    return act * u, ba * np.abs(u) + np.abs(act) * bu + ba * bu + 2.0 ** -24 * np.abs(act * u)


def _check(got, want, b, y_dtype, what=""):
    import torch
    got = got.double().cpu().numpy()
    lo, hi = (torch.from_numpy(v).to(getattr(torch, y_dtype)).double().numpy() for v in (want - b, want + b))
    ok = (lo <= got) & (got <= hi)
    assert np.all(ok), f"{what}{int((~ok).sum())} of {ok.size} outside, the first at {np.argwhere(~ok)[0]}: {got[~ok][0]} not in [{lo[~ok][0]}, {hi[~ok][0]}]"


def _untouched(buf, rows, cols, step, shift):
    import torch
    used = torch.zeros(buf.numel(), dtype=torch.bool, device="cuda")
    used[shift:shift + rows * step].view(rows, step)[:, :cols] = True
    assert torch.isnan(buf[~used]).all(), "written outside the rows"


def _forward(rng, rows, M, K, group, dtype, zeros, glu, exact, y_dtype=None, step=0, shift=0):
    import paper_2305_06942_amd as ebag
    y_dtype = y_dtype or dtype
    plan = ebag.Q4Gemv(M, K, group, _abi(dtype), glu=glu)
    w = Weights(rng, 1, M, K, group, dtype, zeros, exact)
    x = _x(rng, rows, K, dtype, exact, K + step, shift)
    wide = M // 2 if glu else M
    want, b = _want(x.double().cpu().numpy(), w, 0, glu)
    aligned = w.codes.clone()  # and on a boundary, where rows of a multiple of 4 bytes are too
    for codes in (w.codes, aligned):
        y, buf = _strided(rows, wide, y_dtype, wide + step, shift)
        plan.forward(codes, w.scales, w.zeros, x, y)
        _check(y, want, 0 * b if exact else b, y_dtype)
        _untouched(buf, rows, wide, wide + step, shift)
    plan.close()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,M,K,group,zeros", [
    (1, 1, 1, 32, False), (1, 16, 32, 32, True), (2, 17, 33, 64, True), (1, 5, 7, 128, False), (16, 16, 128, 128, True),
    (3, 33, 127, 32, True), (17, 31, 129, 32, False), (1, 100, 256, 64, True), (33, 48, 255, 96, True), (5, 64, 1000, 32, True),
    (12, 19, 2049, 64, False), (64, 40, 512, 256, True), (70, 130, 640, 160, True), (1, 257, 4096, 128, True),
    (130, 65, 384, 8192, True)])
def test_forward_exact(rows, M, K, group, zeros, dtype):
    _forward(np.random.default_rng([51, rows, M, K]), rows, M, K, group, dtype, zeros, 0, True, y_dtype="float32",
             step=3 if M % 2 else 0, shift=K % 3)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("glu", [0, 1])
@pytest.mark.parametrize("rows,M,K,group,zeros", [
    (1, 2, 5, 32, True), (1, 34, 300, 32, False), (4, 64, 1024, 128, True), (19, 130, 777, 64, True),
    (1, 514, 5001, 128, True), (100, 96, 900, 256, False), (300, 260, 1111, 32, True), (257, 128, 2048, 128, False)])
def test_forward(rows, M, K, group, zeros, glu, dtype):
    _forward(np.random.default_rng([52, rows, M, K]), rows, M, K, group, dtype, zeros, glu, False,
             step=5 if K % 2 else 0, shift=K % 2)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("glu", [0, 1])
@pytest.mark.parametrize("group", [64, 128])
@pytest.mark.parametrize("rows,M,K", [(16, 128, 4096), (12, 34, 8200), (5, 512, 12288), (16, 2048, 5000)])
def test_forward_where_a_tile_has_eight_waves(rows, M, K, group, glu, dtype):
    """Few weight rows: the launches that ask for the most LDS."""
    _forward(np.random.default_rng([63, rows, M]), rows, M, K, group, dtype, True, glu, False)


def test_long_rows_and_many_weight_rows():
    rng = np.random.default_rng(53)
    _forward(rng, 1, 48, 70001, 128, "bfloat16", True, 0, False)
    _forward(rng, 2, 20011, 160, 32, "float16", True, 0, True, y_dtype="float32")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,M,K,group,zeros,glu", [
    (400, 4100, 300, 128, True, 0), (389, 4610, 127, 128, False, 0), (400, 4100, 641, 256, False, 1),
    (1000, 4100, 700, 256, True, 0), (1027, 4098, 256, 128, True, 1), (1000, 8200, 333, 32, True, 0), (1010, 8202, 224, 96, False, 1)])
def test_forward_of_many_rows(rows, M, K, group, zeros, glu, dtype):
    """Products large enough for the matrix-product kernel, in both its widths."""
    _forward(np.random.default_rng([60, rows, M, K]), rows, M, K, group, dtype, zeros, glu, False,
             step=5 if K % 2 else 0, shift=K % 2)


@pytest.mark.parametrize("dtype", TYPES)
def test_forward_of_many_rows_exact(dtype):
    rng = np.random.default_rng(61)
    _forward(rng, 420, 4099, 260, 128, dtype, True, 0, True, y_dtype="float32", step=3, shift=1)
    _forward(rng, 1001, 4099, 384, 128, dtype, False, 0, True, y_dtype="float32")
    _forward(rng, 1001, 8199, 130, 64, dtype, True, 0, True, y_dtype="float32")


def _offsets(rng, E, S, kept, empty):
    n = np.zeros(E, dtype=np.int64)
    live = rng.permutation(E)[:max(1, E - empty)]
    np.add.at(n, rng.choice(live, size=kept), 1)
    if kept > 4:
        n[live[0]] += n[live[-1]] if len(live) > 1 else 0
        n[live[-1]] = 0 if len(live) > 1 else n[live[-1]]
    return np.concatenate([[0], np.cumsum(n)]).astype(np.int32)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("E,N,k,M,K,group,zeros,glu,dropped", [
    (1, 1, 1, 16, 64, 32, False, 0, 0), (4, 3, 2, 34, 100, 32, True, 1, 2), (8, 1, 8, 20, 129, 64, True, 0, 0),
    (70, 20, 3, 33, 260, 128, True, 0, 5), (130, 4, 4, 64, 256, 128, False, 1, 0), (5, 60, 2, 50, 300, 64, True, 1, 120),
    (6, 200, 3, 66, 384, 96, True, 0, 17), (3, 700, 2, 258, 500, 128, True, 1, 3), (2, 900, 1, 300, 1030, 32, False, 0, 0)])
def test_experts(E, N, k, M, K, group, zeros, glu, dropped, gather, dtype):
    import torch
    import paper_2305_06942_amd as ebag
    rng = np.random.default_rng([54, E, N, M, K])
    S, wide = N * k, M // 2 if glu else M
    off = _offsets(rng, E, S, S - dropped, E // 4)
    src = rng.permutation(S).astype(np.int32)
    plan = ebag.Q4Gemv(M, K, group, _abi(dtype), experts=E, glu=glu)
    w = Weights(rng, E, M, K, group, dtype, zeros, at=int(rng.integers(0, 4)) if gather else 0)
    x = _x(rng, N if gather else S, K, dtype, False, K + 3, 1)
    x64 = x.double().cpu().numpy()
    rows = x64[src // k] if gather else x64
    if not gather:
        x[off[-1]:] = float("nan")  # dropped rows are not read
    y, buf = _strided(S, wide, dtype, wide + 1, 3)
    plan.experts(w.codes, w.scales, w.zeros, x, torch.from_numpy(off).cuda(), y,
                 src=torch.from_numpy(src).cuda() if gather else None, k=k)
    for e in range(E):
        lo, hi = off[e], off[e + 1]
        if lo < hi:
            _check(y[lo:hi], *_want(rows[lo:hi], w, e, glu), dtype, f"expert {e}: ")
    assert bool((y[off[-1]:] == 0).all())
    _untouched(buf, S, wide, wide + 1, 3)
    plan.close()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("E,N,k,M,K,group,zeros,glu,dropped", [
    (40, 300, 2, 4098, 200, 128, True, 1, 40), (9, 700, 2, 4100, 260, 128, False, 0, 0), (9, 1400, 2, 4098, 161, 32, True, 1, 77),
    (100, 600, 4, 1100, 384, 384, True, 0, 300)])
def test_experts_of_many_rows(E, N, k, M, K, group, zeros, glu, dropped, gather, dtype):
    test_experts(E, N, k, M, K, group, zeros, glu, dropped, gather, dtype)


def test_small_fp16_values_count():
    """fp16 x below its normal range (2^-14) is a sum like any other, in both kernels."""
    import torch
    import paper_2305_06942_amd as ebag
    rng = np.random.default_rng(62)
    for rows, M in ((3, 64), (1000, 4096)):
        K = 256
        plan = ebag.Q4Gemv(M, K, 128, _abi("float16"))
        w = Weights(rng, 1, M, K, 128, "float16", True)
        x = torch.from_numpy(rng.integers(-1000, 1001, size=(rows, K)) * 2.0 ** -24).half().cuda()
        y = torch.empty((rows, M), device="cuda")
        plan.forward(w.codes, w.scales, w.zeros, x, y)
        _check(y, *_want(x.double().cpu().numpy(), w, 0, 0), "float32")
        plan.close()


def test_rows_are_independent_and_infinities_stay_their_own():
    """A row's result is the same bits whatever the other rows of its launch
    shape hold, NaN and infinities among them."""
    import torch
    import paper_2305_06942_amd as ebag
    rng = np.random.default_rng(55)
    M, K = 70, 500
    plan = ebag.Q4Gemv(M, K, 64, _abi("bfloat16"))
    w = Weights(rng, 1, M, K, 64, "bfloat16", True)
    x = torch.from_numpy(rng.standard_normal((11, K))).bfloat16().cuda()
    clean, dirty = torch.empty((11, M), device="cuda"), torch.empty((11, M), device="cuda")
    plan.forward(w.codes, w.scales, w.zeros, x, clean)
    x[4, 100], x[7, 499] = float("inf"), float("nan")
    plan.forward(w.codes, w.scales, w.zeros, x, dirty)
    others = [n for n in range(11) if n not in (4, 7)]
    assert torch.equal(clean[others], dirty[others])
    assert not torch.isfinite(dirty[[4, 7]]).any()
    plan.close()


def test_offsets_and_rows_out_of_range_are_clamped():
    import torch
    import paper_2305_06942_amd as ebag
    rng = np.random.default_rng(56)
    plan = ebag.Q4Gemv(16, 64, 32, _abi("float32"), experts=3)
    w = Weights(rng, 3, 16, 64, 32, "float32", False)
    x = torch.randn((4, 64), device="cuda")
    y = torch.full((8, 16), float("nan"), device="cuda")
    offsets = torch.tensor([0, 3, 2, 1 << 30], dtype=torch.int32, device="cuda")
    src = torch.tensor([0, 2, 4, 6, -1, 1 << 30, 1, 3], dtype=torch.int32, device="cuda")
    plan.experts(w.codes, w.scales, w.zeros, x, offsets, y, src=src, k=2)
    torch.cuda.synchronize()
    assert bool(torch.isfinite(y).all())
    want, b = _want(x[:3].double().cpu().numpy(), w, 0, 0)
    _check(y[:2], want[:2], b[:2], "float32")
    plan.close()


def test_fp32_counts_with_all_its_bits():
    """One column of x is not zero, and its significand needs 24 bits; the
    weight is 1: the product must be x itself."""
    import torch
    import paper_2305_06942_amd as ebag
    M, K = 16, 256
    plan = ebag.Q4Gemv(M, K, 32, _abi("float32"))
    codes = torch.full((1, M, K // 2), 0x99, dtype=torch.uint8, device="cuda")
    scales = torch.ones((1, M, K // 32), device="cuda")
    rng = np.random.default_rng(57)
    rows = 40
    x = torch.zeros((rows, K), device="cuda")
    at = rng.integers(0, K, size=rows)
    v = torch.from_numpy((rng.standard_normal(rows) * 10.0 ** rng.integers(-20, 20, size=rows)).astype(np.float32)).cuda()
    x[torch.arange(rows), torch.from_numpy(at).cuda()] = v
    y = torch.empty((rows, M), device="cuda")
    plan.forward(codes, scales, None, x, y)
    # (16 + 9) x - (16 + 8) x: two sums of 24 bits and their difference, each off by 2^-23 of 25 |x| at most.
    assert bool(((y - v[:, None]).abs() <= 4 * 25 * 2.0 ** -23 * v.abs()[:, None]).all())
    # Without rounding: 16 bits of significand leave 31 x below 2^24 of its last place.
    v = torch.from_numpy(rng.integers(1 << 15, 1 << 16, size=rows).astype(np.float32)).cuda()
    x[torch.arange(rows), torch.from_numpy(at).cuda()] = v
    plan.forward(codes, scales, None, x, y)
    assert torch.equal(y, v[:, None].expand(rows, M))
    plan.close()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("E,M,K,group", [(1, 3, 1, 32), (2, 5, 100, 32), (1, 7, 257, 96), (3, 16, 512, 128), (1, 2, 333, 1024),
                                          (1, 41, 1000, 64), (2, 9, 769, 256), (1, 3, 2500, 1024)])
def test_quantize(E, M, K, group, zeros, dtype):
    import torch
    import paper_2305_06942_amd as ebag
    rng = np.random.default_rng([58, M, K])
    w = rng.standard_normal((E, M, K)) * 10.0 ** rng.integers(-3, 2, size=(E, M, 1))
    w[:, 0, :group] = 0.0          # a group of zeros
    w[:, -1] = np.abs(w[:, -1])    # one sign
    wd = torch.from_numpy(w).to(getattr(torch, dtype))
    groups = -(-K // group)
    plan = ebag.Q4Gemv(M, K, group, _abi(dtype), experts=E)
    codes = torch.full((E, M, (K + 1) // 2), 255, dtype=torch.uint8, device="cuda")
    scales = torch.full((E, M, groups), float("nan"), dtype=wd.dtype, device="cuda")
    z = torch.full((E, M, groups), 77, dtype=torch.uint8, device="cuda") if zeros else None
    plan.quantize(wd.cuda(), codes, scales, z)
    f = wd.float().numpy()
    for g in range(groups):
        part = f[..., g * group:(g + 1) * group]
        lo, hi = np.minimum(part.min(-1), 0), np.maximum(part.max(-1), 0)
        s = (hi - lo) / np.float32(15) if zeros else np.maximum(hi, -lo) / np.float32(7)
        s = torch.from_numpy(s.astype(np.float32)).to(wd.dtype)
        assert torch.equal(scales[..., g].cpu(), s), "scales"
        s = s.float().numpy()
        safe = np.where(s > 0, s, np.float32(1))
        zero = np.full_like(s, 8)
        if zeros:
            zero = np.where(s > 0, np.clip(np.rint(-lo / safe), 0, 15), 0)
            assert np.array_equal(z[..., g].cpu().numpy(), zero), "zeros"
        q = np.where(s[..., None] > 0, np.rint(part / safe[..., None]), 0) + zero[..., None]
        got = codes.cpu().numpy()
        got = np.stack((got & 15, got >> 4), -1).reshape(E, M, -1)
        assert np.array_equal(got[..., g * group:min(K, (g + 1) * group)], np.clip(q, 0, 15)), "codes"
        if K % 2:
            assert not got[..., K].any(), "the last byte's other half"
    plan.close()


def test_graph_replays_and_other_streams():
    import torch
    import paper_2305_06942_amd as ebag
    rng = np.random.default_rng(59)
    E, M, K, S = 4, 128, 512, 24
    plan = ebag.Q4Gemv(M, K, 128, _abi("bfloat16"), experts=E, glu=1)
    w = Weights(rng, E, M, K, 128, "bfloat16", True)
    x = torch.randn((S, K), device="cuda").bfloat16()
    offsets = torch.tensor([0, 3, 3, 20, 24], dtype=torch.int32, device="cuda")
    y, eager = torch.zeros((S, M // 2), device="cuda"), torch.zeros((S, M // 2), device="cuda")
    plan.experts(w.codes, w.scales, w.zeros, x, offsets, y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan.experts(w.codes, w.scales, w.zeros, x, offsets, y)
    side = torch.cuda.Stream()
    for i in range(4):
        x.copy_(torch.randn((S, K), device="cuda"))
        offsets.copy_(torch.tensor([0, i, 10, 10 + i, 24 - i], dtype=torch.int32))
        y.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            plan.experts(w.codes, w.scales, w.zeros, x, offsets, eager)
        side.synchronize()
        assert torch.equal(y, eager)
        assert not i or bool((y[24 - i:] == 0).all())
    plan.close()

"""Products in 8-bit integers where values, streams, strides and sizes are out of the ordinary; bounds as in test_gpu_q8.py."""
import importlib.util
import os

import numpy as np
import pytest

from tests.test_gpu_q8 import Weights, _check, _plan, _rounded, _scratch, _want

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    torch.cuda.set_device(0)
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("glu", [0, 1])
@pytest.mark.parametrize("M,K", [(70, 304), (6000, 136), (40, 9000)])
def test_one_or_two_rows_that_are_not_numbers(M, K, glu, dtype):
    """On 16-byte boundaries, where the product rounds the rows itself."""
    import torch
    rng = np.random.default_rng([94, M, K])
    plan = _plan(M, K, dtype, glu=glu)
    w = Weights(rng, plan, M, K)
    clean = torch.from_numpy(rng.standard_normal((2, K))).to(getattr(torch, dtype)).cuda()
    xq64, xs64 = _rounded(clean.double().cpu().numpy())
    want, b = _want(xq64, xs64.astype(np.float64), w, 0, glu)
    for at, bad in ((0, float("nan")), (K - 1, -float("inf")), (7, float("inf")), (slice(None), 0.0)):
        for rows in (1, 2):
            x = clean[:rows].clone()
            x[0, at] = bad
            y = torch.full((rows, plan.wide), 7.0, device="cuda")
            plan.forward(w.codes, w.scales, x, y, *_scratch(plan, rows))
            assert y[0].eq(0).all() if bad == 0 else y[0].isnan().all()
            _check(y[1:], want[1:rows], b[1:rows], "float32")
    plan.close()


@pytest.mark.parametrize("rows", [1, 2])
@pytest.mark.parametrize("M,K", [(300, 704), (9000, 256)])
def test_one_or_two_rows_captured_and_replayed(rows, M, K):
    import torch
    rng = np.random.default_rng([95, rows, M])
    plan = _plan(M, K, "bfloat16")
    w = Weights(rng, plan, M, K)
    x = torch.empty((rows, K), dtype=torch.bfloat16, device="cuda").normal_()
    y, y2 = (torch.empty((rows, M), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    scratch, other = _scratch(plan, rows), _scratch(plan, rows)
    plan.forward(w.codes, w.scales, x, y, *scratch)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        plan.forward(w.codes, w.scales, x, y, *scratch)
    for _ in range(4):
        x.copy_(torch.from_numpy(rng.standard_normal((rows, K))))
        y.fill_(float("nan"))
        graph.replay()
        plan.forward(w.codes, w.scales, x, y2, *other)
        torch.cuda.synchronize()
        assert torch.equal(y, y2)
    plan.close()


@pytest.mark.parametrize("rows", [2, 40, 900])
def test_two_streams_at_once(rows):
    """Calls of one plan that run at the same time, with scratch memory of their own."""
    import torch
    M, K = 4100, 2048
    plan = _plan(M, K, "float16")
    w = Weights(np.random.default_rng(96), plan, M, K)
    x = [torch.randn((rows, K), device="cuda").to(torch.float16) for _ in range(2)]
    y = [torch.empty((rows, M), dtype=torch.float16, device="cuda") for _ in range(2)]
    scratch = [_scratch(plan, rows) for _ in range(2)]
    for i in range(2):
        plan.forward(w.codes, w.scales, x[i], y[i], *scratch[i])
    want = [v.clone() for v in y]
    for v in y:
        v.fill_(float("nan"))
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(10):
        for i in range(2):
            plan.forward(w.codes, w.scales, x[i], y[i], *scratch[i], stream=streams[i])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(y, want))
    plan.close()


@pytest.mark.parametrize("rows", [2, 60, 700])
def test_rows_far_apart(rows):
    """Offsets of rows of x and y behind 2^32 bytes."""
    import torch
    M, K, step = 130, 136, (1 << 32) // rows
    plan = _plan(M, K, "bfloat16")
    w = Weights(np.random.default_rng(97), plan, M, K)
    x = torch.randn((rows, K), device="cuda").to(torch.bfloat16)
    want = torch.empty((rows, M), dtype=torch.bfloat16, device="cuda")
    scratch = _scratch(plan, rows)
    plan.forward(w.codes, w.scales, x, want, *scratch)
    wide = torch.empty((rows, step), dtype=torch.bfloat16, device="cuda")
    wide[:, :K] = x
    plan.forward(w.codes, w.scales, wide[:, :K], wide[:, 256:256 + M], *scratch)
    assert torch.equal(wide[:, 256:256 + M], want) and torch.equal(wide[:, :K], x)
    plan.close()


def test_more_rows_than_one_launch_has_threads_for():
    """2^26 rows of weights and a few: rounded by more than one launch, codes behind 2^32 bytes."""
    import torch
    M, K = (1 << 26) + 5, 4
    plan = _plan(M, K, "bfloat16")
    w = torch.empty((1, M, K), dtype=torch.bfloat16, device="cuda").normal_()
    codes = torch.full((1, M, plan.pitch), 99, dtype=torch.int8, device="cuda")
    scales = torch.full((1, M), 7.0, device="cuda")
    plan.quantize(w, codes, scales)
    for at in range(0, M, 1 << 23):
        part = w[0, at:at + (1 << 23)].double()
        s = (part.abs().amax(1) / 127).float()
        assert torch.equal(scales[0, at:at + (1 << 23)], s)
        q = torch.round(part / s.double().clamp_min(1e-300)[:, None]).clamp(-127, 127)
        assert torch.equal(codes[0, at:at + (1 << 23), :K].double(), q)
    for rows in (1, 3, 40):
        x = torch.randn((rows, K), device="cuda").to(torch.bfloat16)
        y = torch.full((rows, M), float("nan"), device="cuda")
        xq, xs = _scratch(plan, rows)
        plan.round(x, xq, xs)
        plan.forward(codes, scales, None, y, xq, xs)
        for at in range(0, M, 1 << 23):
            # The sum is exact in fp32 and rounded with the scales' product: 3 steps, and the definition has them in this order.
            sums = xq[:, :K].double() @ codes[0, at:at + (1 << 23), :K].double().t().contiguous()
            want = sums * xs.double()[:, None] * scales[0, at:at + (1 << 23)].double()
            assert bool(((y[:, at:at + (1 << 23)].double() - want).abs() <= want.abs() * 4 * 2.0 ** -24 + 2.0 ** -149).all())
    plan.close()


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("tokens", [1, 24, 500])
def test_a_serving_layer_captured_and_replayed(bits, tokens):
    """Choice, sort, gated products, products and the sum of a token's rows in one graph, every replay against the eager run."""
    import torch
    spec = importlib.util.spec_from_file_location("moe_layer_captured", os.path.join(ROOT, "examples", "moe_layer.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    gate_up, down, x, logits = example.make(tokens, 16, 4, 512, 256)
    layer = example.ServingLayer(gate_up, down, 4, tokens, bits=bits)
    layer(x, logits)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        out = layer(x, logits)
    torch.cuda.current_stream().wait_stream(side)
    for turn in range(4):
        x.copy_(torch.randn_like(x))
        logits.copy_(torch.randn_like(logits))
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        assert torch.equal(got, layer(x, logits)), f"replay {turn}"


VARIANTS = [  # rows, E, M, K, glu, type: a kernel each, between them every one that the choice of kernel has
    (1492, 85, 118, 443, 0, "bfloat16"), (8660, 1, 18, 396, 1, "float16"), (14174, 6, 2, 140, 0, "float32"), (12217, 1, 2, 1, 1, "bfloat16"),
    (1282, 36, 240, 15402, 0, "float16"), (45, 1, 10756, 12023, 1, "bfloat16"), (43685, 7, 2, 18608, 0, "bfloat16"),
    (41197, 1, 2, 17042, 1, "float16"), (58524, 1, 2, 11262, 0, "float32"), (56416, 1, 22, 1, 1, "float32"), (58067, 1, 20, 1, 0, "bfloat16"),
    (54563, 1, 34, 1, 1, "float16"), (33948, 1, 96, 789, 0, "float16"), (44343, 1, 66, 714, 1, "bfloat16"), (51518, 1, 52, 834, 0, "bfloat16"),
    (56569, 3, 120, 1236, 1, "float16"), (20640, 1, 570, 2102, 0, "float16"), (59061, 1, 154, 2604, 1, "bfloat16"),
    (1345, 1, 11456, 2955, 0, "bfloat16"), (1374, 1, 11372, 3459, 1, "float16"), (2300, 3, 9000, 2048, 0, "float32"),
    (64, 1, 60000, 128, 0, "float16"), (35, 15, 3894, 336, 1, "bfloat16"), (77, 17, 2610, 94, 1, "float16")]


@pytest.mark.parametrize("rows,E,M,K,glu,dtype", VARIANTS)
def test_every_kernel_against_64_bits(rows, E, M, K, glu, dtype):
    """The definition on the GPU in 64 bits: the sums are whole numbers below 2^53."""
    import torch
    from tests.test_gpu_q8 import U
    rng = np.random.default_rng([98, rows, M, K])
    gen = torch.Generator(device="cuda").manual_seed(rows + M)
    plan = _plan(M, K, dtype, experts=E, glu=glu)
    codes = torch.randint(-128, 128, (E, M, plan.pitch), dtype=torch.int8, device="cuda", generator=gen)
    scales = (torch.rand((E, M), device="cuda", generator=gen) + 0.5) / (73 * K ** 0.5)
    x = torch.randn((rows, K), device="cuda", generator=gen).to(getattr(torch, dtype))
    xq, xs = _scratch(plan, rows)
    plan.round(x, xq, xs)
    y = torch.full((rows, plan.wide), float("nan"), dtype=x.dtype, device="cuda")
    ends = np.array([0, rows]) if E == 1 else np.concatenate(([0], np.sort(rng.integers(0, rows, size=E - 1)), [rows - 3]))
    if E == 1:
        plan.forward(codes, scales, None, y, xq, xs)
    else:
        plan.experts(codes, scales, None, torch.from_numpy(np.minimum(ends, rows - 3).astype(np.int32)).cuda(), y, xq, xs)
        assert y[rows - 3:].eq(0).all()
    for e in range(E):
        for at in range(int(ends[e]), min(int(ends[e + 1]), rows - 3 if E > 1 else rows), 8192):
            n = slice(at, min(at + 8192, int(ends[e + 1]), rows - 3 if E > 1 else rows))
            want = (xq[n, :K].double() @ codes[e, :, :K].double().t().contiguous()) * xs[n].double()[:, None] * scales[e].double()
            b = 4 * U * want.abs() + 2.0 ** -149
            if glu:
                g, u, bg, bu = want[:, :M // 2], want[:, M // 2:], b[:, :M // 2], b[:, M // 2:]
                act = g / (1 + torch.exp(-g))
                ba = 1.1 * bg + (g.abs() + 8) * 2.0 ** -22 * act.abs()
                want, b = act * u, ba * u.abs() + act.abs() * bu + ba * bu + U * (act * u).abs()
            lo, hi, got = (want - b).to(x.dtype), (want + b).to(x.dtype), y[n]
            ok = (lo <= got) & (got <= hi)
            assert bool(ok.all()), f"{int((~ok).sum())} of {ok.numel()} outside, first {(~ok).nonzero()[0].tolist()} of expert {e}"
    plan.close()


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("M,K,glu", [(300, 700, 0), (3000, 200, 1), (9000, 512, 0), (514, 2048, 1)])
def test_a_row_has_the_same_bits_whatever_rows_are_with_it(M, K, glu, dtype):
    """One row to some thousands go through different kernels; sums are exact and the rest is the same steps."""
    import torch
    plan = _plan(M, K, dtype, glu=glu)
    w = Weights(np.random.default_rng(99), plan, M, K)
    x = torch.randn((5000, K), device="cuda").to(getattr(torch, dtype))
    first = None
    for rows in (5000, 1, 2, 3, 16, 17, 40, 64, 100, 257, 700, 2049):
        y = torch.full((rows, plan.wide), float("nan"), dtype=x.dtype, device="cuda")
        plan.forward(w.codes, w.scales, x[:rows], y, *_scratch(plan, rows))
        first = y if first is None else first
        assert torch.equal(y, first[:rows]), f"{rows} rows"
    plan.close()

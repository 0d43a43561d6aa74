"""One call of a kind in flight per plan: the rule itself without a GPU (built
with g++ against the HIP headers), and the calls that keep to it, on the GPU."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(shutil.which("g++") is None or not os.path.isdir("/opt/rocm/include"),
                    reason="needs g++ and the HIP headers")
def test_the_rule(tmp_path):
    exe = tmp_path / "in_flight_check"
    subprocess.run(["g++", "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                    "-I" + os.path.join(ROOT, "paper_2305_06942_amd", "csrc"), "-I" + os.path.join(ROOT, "include"),
                    os.path.join(ROOT, "tests", "in_flight_check.cpp"), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "bad=0" in r.stdout


def _keep_busy():
    import torch
    a = torch.randn((8192, 8192), device="cuda")
    for _ in range(24):
        a = a @ a * 1e-4


def _capture(fn):
    import torch
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        fn()
    return g


@pytest.mark.gpu
def test_a_capture_does_not_forget_a_sort_in_flight():
    import torch
    import paper_2305_06942_amd as ebag
    torch.cuda.set_device(0)
    N, k, E = 60000, 8, 64
    plan = ebag.MoePerm(N, k, E)
    ids = torch.randint(0, E, (N, k), device="cuda", dtype=torch.int32)
    new = lambda: (torch.zeros(E + 1, dtype=torch.int32, device="cuda"), torch.zeros_like(ids),  # noqa: E731
                   torch.zeros(N * k, dtype=torch.int32, device="cuda"))
    first, second = new(), new()
    first_stream, side = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(first_stream):
        _keep_busy()  # keeps the sort from completing while the others are asked for
        plan.sort(ids, *first)
    done = torch.cuda.Event()
    done.record(first_stream)
    # torch synchronizes where a capture of its own begins, so this one is opened by hand.
    graph = torch.cuda.CUDAGraph()
    capturing = torch.cuda.Stream()
    with torch.cuda.stream(capturing):
        graph.capture_begin()
        plan.sort(ids, *second)
        graph.capture_end()
    assert not done.query(), "the first sort ended before the last one was asked for"
    with pytest.raises(ebag.EbagError, match="sort of this plan is still running"):
        plan.sort(ids, *second, stream=side)
    torch.cuda.synchronize()
    plan.sort(ids, *second, stream=side)
    side.synchronize()
    for a, b in zip(first, second):
        assert torch.equal(a, b)
    plan.close()


@pytest.mark.gpu
def test_a_capture_does_not_forget_a_gemv_in_flight():
    import torch
    import paper_2305_06942_amd as ebag
    torch.cuda.set_device(0)
    M, K = 512, 256
    h = ebag.GemvAR(2, M, [K, K], ebag.EBAG_F32)
    A = [torch.randn((M, K), device="cuda") for _ in range(2)]
    x = [torch.randn(K, device="cuda") for _ in range(2)]
    first, second = ([torch.zeros(M, device="cuda") for _ in range(2)] for _ in range(2))
    first_stream, side, capturing = torch.cuda.Stream(), torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(first_stream):
        _keep_busy()
        h.forward(A, x, first)
    done = torch.cuda.Event()
    done.record(first_stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(capturing):
        graph.capture_begin()
        h.forward(A, x, second)
        graph.capture_end()
    assert not done.query(), "the first forward ended before the last one was asked for"
    with pytest.raises(ebag.EbagError, match="still running on another stream"):
        h.forward(A, x, second, stream=side)
    torch.cuda.synchronize()
    h.forward(A, x, second, stream=side)
    side.synchronize()
    for a, b in zip(first, second):
        assert torch.equal(a, b)
    h.close()

"""GPU tests of calls on several streams at once and of captured ones: every output is filled before both sides, so that one which is not
written shows."""
import torch
import pytest

from paper_2503_17922_b200 import binding as wkv
from test_gpu_operators import Attend, Prompt

pytestmark = pytest.mark.gpu


def outputs(x):
    return [x.out, x.lse, x.w_out] if isinstance(x, Attend) else [x.out, x.lse, x.lse_obs]


def refill(calls):
    for x in calls:
        for t in outputs(x):
            t.fill_(77.0)
    torch.cuda.synchronize()


def same(x, y):
    return torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8))


def several_calls():
    return [Attend("bf16", 8, 2, 128, 64, "pshd", [[5000, 4990], [2100, 700]], [40, 300], True),
            Attend("bf16", 32, 8, 128, 64, "pshd", [[2000] * 8, [1500] * 8], [1, 1], False),
            Attend("f32", 8, 2, 64, 16, "phsd", [[900, 899]], [7], False),
            Prompt("bf16", 8, 2, 128, [2500], "bhnd", 4), Prompt("f32", 4, 2, 64, [700, 3], "packed", 4)]


def test_every_output_of_calls_on_several_streams():
    calls = several_calls()
    refill(calls)
    for x in calls:
        x.run()
    torch.cuda.synchronize()
    alone = [[t.clone() for t in outputs(x)] for x in calls]
    streams = [torch.cuda.Stream() for _ in calls]
    for _ in range(5):
        refill(calls)
        for x, s in zip(calls, streams):
            with torch.cuda.stream(s):
                x.run()
        torch.cuda.synchronize()
        for x, want in zip(calls, alone):
            assert all(same(t, w) for t, w in zip(outputs(x), want))


def test_every_output_of_captured_calls():
    calls = several_calls()
    rope, turned = wkv.Rope(64), torch.empty_like(calls[3].q)
    lengths = [x.lengths.cuda() for x in calls[:3]]

    def step():
        for x, n in zip(calls[:3], lengths):
            wkv.wkv_attend_paged(x.cache, x.q, x.c.k[0], x.c.v[0], n, x.out, x.ws, lse=x.lse, weights_in=x.w_in, weights_out=x.w_out)
        wkv.wkv_rotate_prompt(calls[3].prob, rope, calls[3].q, None, turned, None)
        for p in calls[3:]:
            p.run()
    refill(calls)
    turned.fill_(77.0)
    step()
    torch.cuda.synchronize()
    want = [[t.clone() for t in outputs(x)] for x in calls] + [[turned.clone()]]
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            step()
    for _ in range(3):
        refill(calls)
        turned.fill_(77.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for got, w in zip([outputs(x) for x in calls] + [[turned]], want):
            assert all(same(a, b) for a, b in zip(got, w))
    for x in calls[:3]:
        assert wkv.device_status(x.ws) == 0


def test_two_graphs_that_share_a_workspace_in_turn():
    """One after the other on one stream, a workspace serves calls of one description in two graphs."""
    a = Attend("bf16", 8, 2, 128, 64, "phsd", [[3000, 2990]], [40], False)
    b = Attend("bf16", 8, 2, 128, 64, "phsd", [[2500, 100]], [40], False, seed=2, max_pages=a.c.max_pages)
    assert a.cache.workspace_bytes == b.cache.workspace_bytes
    lengths = [x.lengths.cuda() for x in (a, b)]
    call = lambda x, n: wkv.wkv_attend_paged(x.cache, x.q, x.c.k[0], x.c.v[0], n, x.out, a.ws, lse=x.lse, weights_in=x.w_in, weights_out=x.w_out)
    refill((a, b))
    call(a, lengths[0])
    call(b, lengths[1])
    torch.cuda.synchronize()
    want = [[t.clone() for t in outputs(x)] for x in (a, b)]
    side, graphs = torch.cuda.Stream(), []
    with torch.cuda.stream(side):
        for x, n in zip((a, b), lengths):
            graphs.append(torch.cuda.CUDAGraph())
            with torch.cuda.graph(graphs[-1], stream=side):
                call(x, n)
    refill((a, b))
    with torch.cuda.stream(side):
        for g in (graphs[0], graphs[1], graphs[1], graphs[0]):
            g.replay()
    torch.cuda.synchronize()
    for x, w in zip((a, b), want):
        assert all(same(s, t) for s, t in zip(outputs(x), w))


def test_the_attention_kernels_wait_ends(tmp_path):
    """For a barrier that nobody arrives at, after its limit, in all warps of the block, and the context goes on."""
    import ctypes
    import os
    import subprocess
    from paper_2503_17922_b200 import build
    so = str(tmp_path / "libwaits.so")
    subprocess.check_call([build._nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-Xcompiler", "-fPIC", "-shared", "-I", build.CSRC,
                           "-o", so, os.path.join(os.path.dirname(os.path.abspath(__file__)), "warp_wait.cu")])
    result, ns = torch.full((128,), -1, dtype=torch.int32, device="cuda"), torch.zeros(128, dtype=torch.int64, device="cuda")
    abort = torch.full((1,), -1, dtype=torch.int32, device="cuda")
    ptr = lambda t: ctypes.c_void_p(t.data_ptr())
    assert ctypes.CDLL(so).run_waits(ptr(result), ptr(ns), ptr(abort), ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)) == 0
    torch.cuda.synchronize()
    assert (result == 1).all() and int(abort) == 1                        # the complete barrier is seen, the other is not
    assert 0.5e9 < int(ns.min()) and int(ns.max()) < 3e9                  # the limit is one second
    a = Attend("bf16", 8, 2, 128, 16, "phsd", [[300, 299]], [20], False)
    a.run()
    a.check()

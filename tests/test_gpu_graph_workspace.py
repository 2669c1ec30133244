"""Calls recorded in a graph without a workspace of the caller: each graph has its own, which
no later call replaces and each replay clears."""

import pytest
import torch

from synth import make_problem
from test_gpu_layer import Step, log

pytestmark = pytest.mark.gpu


def attend(fq, kind, kv_lens, seed, q_lens=None):
    st = Step(fq, kind, 128, 8, 2, 64, q_lens or [1] * len(kv_lens), kv_lens, seed=seed)
    c = fq.fq_paged_attention_launch(8, st.q.shape[0], st.cache, st.batch)
    assert c["split"] > 1
    return (lambda: fq.fq_paged_attention(st.q, st.cache, st.batch)), c["partial_kib"]


def matmul(fq, M, K, N, seed):
    prob = make_problem(M, K, N, frac=0.01, seed=seed)
    args = (*fq.to_device(prob), fq.TileCOODevice(fq.fq_pack_tile_coo(K, N, prob.k, prob.n, prob.v)))
    c = fq.fq_launch_kernel(M, K, N, args[-1])
    assert c["split_k"] > 1
    return (lambda: fq.fq_w4a16_outlier_matmul(*args)), c["partial_kib"]


def record(call, stream):
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=stream):
        out = call()
    return g, out


@pytest.mark.parametrize("warm", [False, True], ids=["cold", "warm"])
@pytest.mark.parametrize("what", ["attention_rows", "attention_tiles", "matmul"])
def test_graphs_of_one_stream_and_a_larger_call(gpu_lib, what, warm):
    fq = gpu_lib
    log(f"graphs {what} warm={warm}")
    if what == "attention_rows":
        calls = [attend(fq, "int8", [3000, 700], 1), attend(fq, "bf16", [5000], 2)]
        more = attend(fq, "int8", [9000] * 6, 3)
    elif what == "attention_tiles":
        calls = [attend(fq, "int8", [3000], 1, [300]), attend(fq, "bf16", [6000], 2, [270])]
        more = attend(fq, "int4", [16000], 3, [400])
    else:
        calls = [matmul(fq, 8, 14336, 256, 1), matmul(fq, 16, 14336, 512, 2)]
        more = matmul(fq, 16, 14336, 4096, 3)
    assert more[1] > max(c[1] for c in calls)
    calls, more = [c[0] for c in calls], more[0]
    want, most = [c() for c in calls], more()
    stream = torch.cuda.Stream()
    # streams come from a pool: what earlier users of this one kept is put back at the end
    key = (torch.cuda.current_device(), stream.cuda_stream)
    before = fq._workspaces.pop(key, None)
    try:
        torch.cuda.synchronize()
        if warm:
            with torch.cuda.stream(stream):
                for c in calls:
                    c()
            torch.cuda.synchronize()
        graphs = [record(c, stream) for c in calls]
        with torch.cuda.stream(stream):
            grown = more()                        # replaces the stream's kept workspace
        torch.cuda.synchronize()
        assert torch.equal(grown, most)
        others = [torch.full((1 << 22,), 3, dtype=torch.int32, device="cuda") for _ in range(8)]
        for r in range(3):
            for i in (1, 0, 1):                   # the second graph first
                g, out = graphs[i]
                out.fill_(float("nan"))
                torch.cuda.synchronize()
                g.replay()
                torch.cuda.synchronize()
                assert torch.equal(out, want[i]), (r, i)
                with torch.cuda.stream(stream):
                    assert torch.equal(more(), most)
                    assert torch.equal(calls[i](), want[i])
                torch.cuda.synchronize()
        assert all((t == 3).all() for t in others)
    finally:
        fq._workspaces.pop(key, None)
        if before is not None:
            fq._workspaces[key] = before


def test_calls_of_one_graph_share_a_workspace(gpu_lib):
    """Several calls in one graph, on two streams of its own."""
    fq = gpu_lib
    log("one graph, several calls")
    calls = [attend(fq, "int8", [3000, 700], 1)[0], attend(fq, "bf16", [5000], 2)[0], matmul(fq, 8, 14336, 256, 1)[0]]
    want = [c() for c in calls]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        here = torch.cuda.current_stream()
        first = [c() for c in calls]
        side.wait_stream(here)
        with torch.cuda.stream(side):
            second = [c() for c in calls]
        third = [c() for c in calls]
        here.wait_stream(side)
    for r in range(3):
        for o in (first, second, third):
            for t in o:
                t.fill_(float("nan"))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for o in (first, second, third):
            for t, w in zip(o, want):
                assert torch.equal(t, w), r

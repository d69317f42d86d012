"""The whole step (compaction, forward, backward) captured in a HIP graph: the library
allocates nothing, never synchronises and uses only kernels (no memset nodes), so a caller may
capture it.  Replays are interleaved with eager work and every replay is compared with the
eager result."""
import pytest
import torch

from paper_2503_21817_amd import binding as B
from paper_2503_21817_amd import workloads as W
from helpers import Problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("r_host", [True, False], ids=["R-host", "R-device"])
def test_graph_replays_match_eager(r_host):
    w = W.small(C=512, I=1368, visual=(300, 411), text=(20, 35), keep=(130, 212), seed=61, name="graph")
    p = Problem(w)
    T, R, C, I = w.T, w.R, w.C, w.I
    bufs = B.SkipFFNBuffers(T, R if r_host else T, C, I, training=True)
    dws = [torch.zeros((I, C), dtype=torch.bfloat16, device="cuda"),
           torch.zeros((I, C), dtype=torch.bfloat16, device="cuda"),
           torch.zeros((C, I), dtype=torch.bfloat16, device="cuda")]
    dgain = torch.zeros(C, dtype=torch.float32, device="cuda")
    hidden = p.d_hidden.clone()
    grad = p.d_grad.clone()
    out = torch.empty_like(hidden)
    gh = torch.empty_like(grad)

    def step():
        B.skipffn_compact(p.d_mask, bufs.idx, bufs.num_retained, None, bufs.compact_ws)
        B.skipffn_forward(hidden, out, bufs.idx, R if r_host else None, p.d_wg, p.d_wu, p.d_wd,
                          eps=w.eps, num_retained=bufs.num_retained, saved=bufs.saved,
                          workspace=bufs.fwd_ws)
        B.skipffn_backward(grad, gh, bufs.idx, R if r_host else None, p.d_wg, p.d_wu, p.d_wd,
                           bufs.saved, *dws, eps=w.eps, num_retained=bufs.num_retained,
                           workspace=bufs.bwd_ws, d_rms_gain=dgain)

    step()                                   # eager reference (also the one-time kernel set-up)
    torch.cuda.synchronize()
    ref = [t.clone() for t in (out, gh, *dws, dgain)]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        step()                               # warm-up on the capture stream
        side.synchronize()
        with torch.cuda.graph(g, stream=side):
            step()
    torch.cuda.synchronize()

    for rep in range(4):
        for t in (out, gh, *dws, dgain):     # eager work between replays: poison the outputs
            t.fill_(float("nan") if t.is_floating_point() else 0)
        bufs.idx.fill_(-1)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip((out, gh, *dws, dgain), ref):
            assert torch.equal(a.view(torch.int16) if a.dtype == torch.bfloat16 else a,
                               b.view(torch.int16) if b.dtype == torch.bfloat16 else b), f"replay {rep}"


def test_attention_calls_replay_from_a_graph():
    """Forward, backward and single tokens captured once and replayed with eager work between the replays: the bits of the eager
    calls, from two graphs that share their workspaces too."""
    import numpy as np
    T, Hq, Hkv, D = 300, 8, 2, 128
    gen = torch.Generator(device="cuda").manual_seed(3)
    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda").to(torch.bfloat16)
    def ints(*v):
        return torch.tensor(v, dtype=torch.int32, device="cuda")
    def room(n):
        return torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")
    q, k, v, g = normal(T, Hq, D), normal(3000, Hkv, D), normal(3000, Hkv, D), normal(T, Hq, D)
    seg_q, seg_k = ints(0, 20, T), ints(0, 2500, 3000)
    few_q, few_k = ints(0, 20), ints(0, 2500)                         # parts of keys, and the kernel that joins them
    out, few, step = torch.zeros_like(q), torch.zeros_like(q[:20]), torch.zeros_like(q[:4])
    grads = [torch.zeros_like(t) for t in (q, k, v)]
    saved, bws = room(B.skipffn_attn_saved_bytes(T, Hq)), room(B.skipffn_attn_backward_workspace_bytes(T, 3000, 2, Hq, Hkv, D))
    shared = room(max(B.skipffn_attn_forward_workspace_bytes(T, 3000, 2, Hq, Hkv, D), B.skipffn_attn_forward_workspace_bytes(20, 2500, 1, Hq, Hkv, D),
                      B.skipffn_attn_decode_workspace_bytes(4, 2, Hq, Hkv, D, 3000, 16)))
    own, lens, off = normal(2, 4, 16, Hkv, D), ints(3, 16, 0, 9), ints(0, 3, 4)

    def prompts():
        B.skipffn_attn_forward(q, k, v, out, seg_q, seg_k, saved=saved, workspace=shared)
        B.skipffn_attn_backward(q, k, v, out, g, seg_q, seg_k, saved, *grads, workspace=bws)

    def tokens():
        B.skipffn_attn_forward(q[:20], k[:2500], v[:2500], few, few_q, few_k, workspace=shared)
        B.skipffn_attn_decode(q[:4], k, v, seg_k, off, own[0], own[1], lens, step, workspace=shared)

    results = [out, few, step, *grads]
    prompts()
    tokens()
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for graph, work in zip(graphs, (prompts, tokens)):
        with torch.cuda.graph(graph):
            work()
    for turn in range(4):
        for t in (q, k, v, g, own):
            t.copy_(normal(*t.shape))                                # new inputs in the same memory
        prompts()
        tokens()
        torch.cuda.synchronize()
        want = [t.clone() for t in results]
        for t in results:
            t.zero_()
        saved.fill_(0xA5)
        bws.fill_(0xA5)
        shared.fill_(0xA5)
        graphs[turn % 2].replay()
        graphs[1 - turn % 2].replay()
        torch.cuda.synchronize()
        for name, a, b in zip("out few step dq dk dv".split(), results, want):
            assert torch.equal(a, b), (turn, name)


def test_attention_on_another_stream_than_the_default():
    T, H, D = 130, 4, 64
    side = torch.cuda.Stream()
    q = torch.randn(T, H, D, device="cuda").to(torch.bfloat16)
    seg = torch.tensor([0, T], dtype=torch.int32, device="cuda")
    a, b = torch.zeros_like(q), torch.zeros_like(q)
    B.skipffn_attn_forward(q, q, q, a, seg)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        late = q * 1                                                 # the call has to wait for this
        B.skipffn_attn_forward(late, late, late, b, seg)
    side.synchronize()
    torch.cuda.synchronize()
    assert torch.equal(a, b)


def test_attention_calls_at_once_on_two_streams():
    """Two calls whose kernels may overlap, each with its own workspace, give what they give one after the other."""
    Hq, Hkv, D, Tk = 8, 2, 128, 3000
    def room(n):
        return torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")
    seg_q, seg_k = torch.tensor([0, 7, 30], dtype=torch.int32, device="cuda"), torch.tensor([0, 1200, Tk], dtype=torch.int32, device="cuda")
    jobs = []
    for _ in range(2):
        q, k, v = (torch.randn(t, h, D, device="cuda").to(torch.bfloat16) for t, h in ((30, Hq), (Tk, Hkv), (Tk, Hkv)))
        jobs.append((q, k, v, torch.zeros_like(q), room(B.skipffn_attn_forward_workspace_bytes(30, Tk, 2, Hq, Hkv, D))))
    assert jobs[0][4].numel() > 16
    for q, k, v, out, ws in jobs:
        B.skipffn_attn_forward(q, k, v, out, seg_q, seg_k, workspace=ws)
    torch.cuda.synchronize()
    want = [job[3].clone() for job in jobs]
    streams = [torch.cuda.Stream() for _ in jobs]
    for _ in range(20):
        for job in jobs:
            job[3].zero_()
        for s in streams:
            s.wait_stream(torch.cuda.current_stream())
        for s, (q, k, v, out, ws) in zip(streams, jobs):
            with torch.cuda.stream(s):
                B.skipffn_attn_forward(q, k, v, out, seg_q, seg_k, workspace=ws)
        for s in streams:
            torch.cuda.current_stream().wait_stream(s)
        torch.cuda.synchronize()
        assert all(torch.equal(job[3], w) for job, w in zip(jobs, want))

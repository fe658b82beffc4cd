"""Workspaces made on one stream and used on another."""

import pytest

import mm_reference as ref
from test_gpu_kv_replays import check, setup
from test_gpu_mm import operands, rows

pytestmark = pytest.mark.gpu


def test_made_on_one_stream_used_on_another(fsb, cuda):
    """The constructor's fill is done when it returns, however much its stream has ahead of it: a backward pass on another stream
    keeps dg and du in that memory between its kernels."""
    torch = cuda
    T, K, N = 700, 520, 1003
    x, w, _, _, dt = operands(torch, "bfloat16", T, K, N, 2, 1)
    dy = rows(torch, T, N, dt, 3)[0]
    outs = [rows(torch, n, K, dt, 0)[0] for n in (T, N, N)]
    one, other = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(one):
        torch.cuda._sleep(20_000_000)
        work = fsb.MmWorkspace(T, K, N, backward=True)
        assert one.query()
    fsb.fs_gated_ff_backward(x, *w, dy, *outs, workspace=work, stream=other)
    fsb.fs_mm_check(work, stream=other)
    for o, want in zip(outs, ref.gated_backward(x, *w, dy)):
        ref.near(o, want)


def test_made_within_a_capture(fsb, cuda):
    torch = cuda
    T, K, N = 200, 136, 300
    x, w, _, _, dt = operands(torch, "bfloat16", T, K, N, 2, 1)
    dy = rows(torch, T, N, dt, 3)[0]
    outs = [rows(torch, n, K, dt, 0)[0] for n in (T, N, N)]
    fsb.fs_gated_ff_backward(x, *w, dy, *outs, workspace=fsb.MmWorkspace(T, K, N, backward=True))  # (what a first call sets up)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work = fsb.MmWorkspace(T, K, N, backward=True)
        fsb.fs_gated_ff_backward(x, *w, dy, *outs, workspace=work)
    for seed in range(2):
        x.copy_(rows(torch, T, K, dt, 20 + seed)[0])
        graph.replay()
        for o, want in zip(outs, ref.gated_backward(x, *w, dy)):
            ref.near(o, want)
    fsb.fs_mm_check(work)


def test_the_cache_operators(fsb, cuda):
    """Tickets and parts of results of a cache that is read in parts: the fill is done when the constructor returns."""
    torch = cuda
    d, cache, b, q, _ = setup(torch, fsb, 1, 2, 2, 8, 128, 32, 4000)
    out = torch.full_like(q, 7.0)
    one, other = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(one):
        torch.cuda._sleep(20_000_000)
        work = fsb.KvWorkspace(cache, b, 16)
        assert one.query()
    fsb.fs_kv_attend(cache, b, q, out, 0.1, workspace=work, stream=other)
    fsb.fs_kv_check(work, stream=other)
    check(out, q, d, d["length"], d["q_start"], 0.1)

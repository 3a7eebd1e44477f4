"""Workspaces in use: a captured step outlives the sparse update's outgrown one, graphs of layer norm's backward run beside each
other and beside eager calls, and one for the largest batch does for all."""
import pytest
import torch

from paper_2103_00686_amd import binding as B
from paper_2103_00686_amd.hotpath import HotPath
from test_gpu_norm_step import _batch, _tables

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("pooling", [B.FAE_POOL_SUM, B.FAE_POOL_MEAN])
def test_a_captured_step_outlives_the_workspaces(pooling):
    rows, S, lr, dim = [500, 90, 40], 200, 0.05, 32
    st = torch.cuda.Stream()
    hp = _tables(rows, dim, st.cuda_stream)
    hb, big = _batch(rows, S, 1, 5), _batch(rows, 60_000, 2, 5)
    gy = torch.randn((S, 3, dim), device="cuda")
    torch.cuda.synchronize()
    start = [w.clone() for w in hp.hotW]

    def step():
        pooled, y = hp.forward_norm(hb, pooling=pooling)
        return (y, *hp.backward_norm_sgd(hb, pooled, gy, lr, pooling=pooling))
    first = step()
    hp.sync()
    want = [t.clone() for t in (*first, *hp.hotW)]
    torch.cuda.synchronize()
    small = hp.bwd_workspace(hb).data_ptr()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        got = step()
    torch.cuda.synchronize()
    pooled, y = hp.forward_norm(big, pooling=pooling)
    hp.sync()
    hp.backward_norm_sgd(big, pooled, torch.ones_like(y), lr, pooling=pooling)
    hp.sync()
    assert hp.bwd_workspace(big).data_ptr() != small
    fill = [torch.full((1 << 20,), float("nan"), device="cuda") for _ in range(64)]
    for _ in range(3):
        for w, s in zip(hp.hotW, start):
            w.copy_(s)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip((*got, *hp.hotW), want):
            assert torch.equal(a, b)
    assert all(bool(torch.isnan(f).all()) for f in fill)


@pytest.mark.parametrize("forked", [False, True])
def test_graphs_beside_each_other(forked):
    """Two graphs of one HotPath on two streams, an eager call between them.  forked: the capture starts on another stream than
    the HotPath's, which joins it."""
    st, other = torch.cuda.Stream(), torch.cuda.Stream()
    hp = HotPath([1], 4, stream=st.cuda_stream)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    shapes = [(3000, 26, 64), (2000, 1, 1000), (5000, 3, 100)]
    x, gy = ([torch.randn(s, device="cuda", generator=gen) for s in shapes] for _ in range(2))
    torch.cuda.synchronize()
    want = [hp.layer_norm_backward(x[i], gy[i]) for i in range(3)]
    hp.sync()
    graphs, got = [], []
    for i in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[i], stream=other if forked else st):
            if forked:
                st.wait_stream(other)
            got.append([hp.layer_norm_backward(x[i], gy[i]) for _ in range(4)])
            if forked:
                other.wait_stream(st)
    lanes = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        for outs in got:
            for out in outs:
                for t in out:
                    t.fill_(float("nan"))
        torch.cuda.synchronize()
        for graph, lane in zip(graphs, lanes):
            with torch.cuda.stream(lane):
                graph.replay()
        eager = hp.layer_norm_backward(x[2], gy[2])
        torch.cuda.synchronize()
        for i in range(2):
            for out in got[i]:
                for a, b in zip(out, want[i]):
                    assert torch.equal(a, b)
        for a, b in zip(eager, want[2]):
            assert torch.equal(a, b)


@pytest.mark.parametrize("parts,width,rows", [(1, 64, [16537, 16213, 9000, 70]), (13, 64, [1283, 1258, 40]), (4, 100, [2049, 2009, 300]), (1, 2000, [3000, 900, 5])])
def test_the_largest_batch_s_workspace_for_all(parts, width, rows):
    """Smaller batches in it leave what lies behind it as it was, and have the results of a call with their own."""
    hp = HotPath([1], 4)
    need = B.fae_layer_norm_bwd_workspace_bytes(B.Norm(rows[0], parts, width))
    buf = torch.full((need + 4096,), 0x5A, dtype=torch.uint8, device="cuda")
    for n in rows:
        x, gy = torch.randn((2, n, parts, width), device="cuda")
        want = hp.layer_norm_backward(x, gy)
        gx, dg, db = torch.empty_like(x), *torch.empty((2, parts, width), device="cuda")
        B.fae_layer_norm_bwd(hp.ctx, B.Norm(n, parts, width), x, gy, gx, dg, db, buf[:need])
        hp.sync()
        for a, b in zip((gx, dg, db), want):
            assert torch.equal(a, b)
        assert bool((buf[need:] == 0x5A).all())

"""A whole step as it is used: pooled forward, layer norm with dropout, back through both, sparse SGD on the hot tables, all
against 64 bits from the tables and the lookups alone; eager, and captured into a graph."""
import numpy as np
import pytest
import torch

import rows_ref as R
from paper_2103_00686_amd import binding as B
from paper_2103_00686_amd.hotpath import HotBatch, HotPath

pytestmark = pytest.mark.gpu

EPS = 1e-5


def _batch(rows, S, seed, longest):
    rng = np.random.default_rng(seed)
    slots, offs, nl = [], [], []
    for z, r in enumerate(rows):
        ln = np.ones(S, dtype=np.int64) if z % 2 == 0 else rng.integers(0, longest + 1, S)
        slots.append(torch.from_numpy(rng.integers(0, r, int(ln.sum()), dtype=np.int32)).cuda())
        offs.append(None if z % 2 == 0 else torch.from_numpy(np.concatenate([[0], np.cumsum(ln)]).astype(np.int32)).cuda())
        nl.append(int(ln.sum()))
    return HotBatch(S, slots, offs, nl)


def _tables(rows, dim, stream=None):
    hp = HotPath(rows, dim, stream=stream)
    hp.alloc_counts()
    hp.build([0] * len(rows), rows, seed=3)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(7)
    for w in hp.hotW:
        w.normal_(generator=gen)
    return hp


def _pool(w, hb, z):
    n = hb.offsets[z].long().diff() if hb.offsets[z] is not None else torch.ones(hb.n_samples, dtype=torch.int64, device="cuda")
    seg = torch.repeat_interleave(torch.arange(hb.n_samples, device="cuda"), n)
    return torch.zeros((hb.n_samples, w.shape[1]), dtype=torch.float64, device="cuda").index_add_(0, seg, w[hb.slots[z].long()]), seg


@pytest.mark.parametrize("dim", [16, 50, 64])
@pytest.mark.parametrize("p", [0.0, 0.2])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_step(dim, p, dtype):
    rows, S, lr = [500, 90, 40], 333, 0.01
    hp, hb = _tables(rows, dim), _batch(rows, S, dim, 6)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(dim)
    gamma, beta = (torch.randn((3, dim), device="cuda", generator=gen) for _ in range(2))
    drop = B.Drop(p, 11, 5) if p > 0 else None
    w0 = [w.clone() for w in hp.hotW]
    pooled, y = hp.forward_norm(hb, gamma, beta, EPS, drop, dtype)
    x = pooled.clone()
    gy = torch.randn(y.shape, device="cuda", generator=gen).to(dtype)
    dgamma, dbeta = hp.backward_norm_sgd(hb, pooled, gy, lr, gamma, EPS, drop)
    hp.sync()
    keep, scale = (None, 1.0) if p == 0 else R.keep_and_scale(S * 3, dim, p, 11, 5)
    ref = R.NormRef(x, gamma, beta, EPS, None if keep is None else keep.reshape(x.shape).cuda(), scale)
    R.assert_within(y, *ref.forward(dtype), "y")
    (gx, dg, db), (tx, tg, tb) = ref.backward(gy, torch.float32)
    R.assert_within(pooled, gx, tx, "gradient of the pooled rows")
    R.assert_within(dgamma, dg, tg, "dgamma")
    R.assert_within(dbeta, db, tb, "dbeta")
    for z in range(3):
        px, seg = _pool(w0[z].double(), hb, z)
        mag, _ = _pool(w0[z].double().abs(), hb, z)
        assert bool(((x[:, z].double() - px).abs() <= 8 * R.U * mag).all())  # six rows of a bag
        idx = hb.slots[z].long()
        G = torch.zeros_like(w0[z], dtype=torch.float64).index_add_(0, idx, gx[seg, z])
        mag = torch.zeros_like(G).index_add_(0, idx, gx[seg, z].abs())
        tol = torch.zeros_like(G).index_add_(0, idx, tx[seg, z])
        n = torch.zeros(rows[z], dtype=torch.float64, device="cuda").index_add_(0, idx, torch.ones(len(idx), dtype=torch.float64, device="cuda"))
        want = w0[z].double() - lr * G  # lr * (the allowed error of gx and a sum's roundings), lr's own rounding and two of the update
        R.assert_within(hp.hotW[z], want, lr * (tol + (n[:, None] + 3) * R.U * mag) + 2 * R.U * want.abs() + 1e-30, f"table {z}")


@pytest.mark.parametrize("dim,p", [(64, 0.1), (20, 0.0)])
def test_step_in_a_graph(dim, p):
    """The step as one graph: each replay moves the tables and draws a new mask by the counter on the device, as eager steps do."""
    rows, S, lr = [500, 90, 40, 7], 200, 0.05
    st = torch.cuda.Stream()
    hp = _tables(rows, dim, st.cuda_stream)
    hb = _batch(rows, S, 1, 5)
    nt = len(rows)
    gamma, beta = torch.randn((2, nt, dim), device="cuda")
    counter = torch.zeros(1, dtype=torch.int64, device="cuda")
    gy = torch.randn((S, nt, dim), device="cuda")
    x, y, gx = (torch.empty((S, nt, dim), device="cuda") for _ in range(3))
    dg, db = torch.empty((2, nt, dim), device="cuda")
    norm, drop = B.Norm(S, nt, dim, gamma, beta, EPS), B.Drop(p, 3, 0, counter) if p > 0 else None
    fwd, bwd = hp.prepare_layer_norm(norm, x, y, drop), hp.prepare_layer_norm_backward(norm, x, gy, gx, dg, db, drop)
    hp.bwd_workspace(hb)
    torch.cuda.synchronize()
    start = [w.clone() for w in hp.hotW]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        hp.forward(hb, out=x)
        fwd()
        bwd()
        hp.backward_sgd(hb, gx, lr)
        counter += 1
    torch.cuda.synchronize()
    for w, s in zip(hp.hotW, start):
        w.copy_(s)
    counter.zero_()
    seen = []
    for _ in range(4):
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        seen.append([y.clone(), dg.clone(), db.clone()] + [w.clone() for w in hp.hotW])
    for w, s in zip(hp.hotW, start):
        w.copy_(s)
    torch.cuda.synchronize()
    for i in range(4):
        d = B.Drop(p, 3, i) if p > 0 else None
        pooled, yy = hp.forward_norm(hb, gamma, beta, EPS, d)
        gg, bb = hp.backward_norm_sgd(hb, pooled, gy, lr, gamma, EPS, d)
        hp.sync()
        for a, b in zip(seen[i], [yy, gg, bb] + hp.hotW):
            assert torch.equal(a, b)


def test_two_at_once():
    """Two programs' steps on two streams, queued in turn without waiting: each has its own workspace."""
    streams = [torch.cuda.Stream() for _ in range(2)]
    hps = [HotPath([1], 4, stream=st.cuda_stream) for st in streams]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    shapes = [(3000, 26, 64), (2000, 1, 1000)]
    x = [torch.randn(sh, device="cuda", generator=gen) for sh in shapes]
    gy = [torch.randn(sh, device="cuda", generator=gen) for sh in shapes]
    gamma = [torch.randn(sh[1:], device="cuda", generator=gen) for sh in shapes]
    torch.cuda.synchronize()  # the tensors were made on another stream than the calls run on, and the results are read on it
    want = [hps[i].layer_norm_backward(x[i], gy[i], gamma[i]) for i in range(2)]
    torch.cuda.synchronize()
    outs = [[[torch.full_like(t, float("nan")) for t in want[i]] for _ in range(8)] for i in range(2)]
    torch.cuda.synchronize()
    calls = [[hps[i].prepare_layer_norm_backward(B.Norm(*shapes[i], gamma[i]), x[i], gy[i], *o) for o in outs[i]] for i in range(2)]
    for a, b in zip(*calls):
        a()
        b()
    torch.cuda.synchronize()
    for i in range(2):
        for o in outs[i]:
            for a, b in zip(o, want[i]):
                assert torch.equal(a, b.reshape(a.shape))


def test_a_captured_step_outlives_its_workspace():
    """A larger call behind the capture needs a larger workspace: the graph still has the one it was captured with."""
    st = torch.cuda.Stream()
    hp = HotPath([1], 4, stream=st.cuda_stream)
    x, gy = torch.randn((2, 700, 3, 40), device="cuda")
    torch.cuda.synchronize()
    want = hp.layer_norm_backward(x, gy)
    hp.sync()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        got = hp.layer_norm_backward(x, gy)
    big = torch.randn((20000, 1, 2000), device="cuda")
    torch.cuda.synchronize()
    hp.layer_norm_backward(big, big)
    hp.sync()
    fill = [torch.full((1 << 20,), float("nan"), device="cuda") for _ in range(64)]
    for _ in range(3):
        for t in got:
            t.fill_(0.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)
    assert all(bool(torch.isnan(f).all()) for f in fill)

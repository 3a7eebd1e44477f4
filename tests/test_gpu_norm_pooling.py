"""The step through layer norm with mean pooling: bags of several lengths, some empty, against 64 bits from the tables and
the lookups alone, eager and in a graph.  Sum pooling through the same arguments is the plain step."""
import pytest
import torch

import rows_ref as R
from paper_2103_00686_amd import binding as B
from test_gpu_norm_step import EPS, _batch, _pool, _tables

pytestmark = pytest.mark.gpu


def _lengths(hb, z):
    if hb.offsets[z] is None:
        return torch.ones(hb.n_samples, dtype=torch.float64, device="cuda")
    return hb.offsets[z].long().diff().double()


@pytest.mark.parametrize("dim", [16, 50, 64])
@pytest.mark.parametrize("p", [0.0, 0.2])
def test_step_with_mean_pooling(dim, p):
    rows, S, lr = [500, 90, 40], 333, 0.01
    hp, hb = _tables(rows, dim), _batch(rows, S, dim, 6)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(dim)
    gamma, beta = (torch.randn((3, dim), device="cuda", generator=gen) for _ in range(2))
    drop = B.Drop(p, 11, 5) if p > 0 else None
    w0 = [w.clone() for w in hp.hotW]
    pooled, y = hp.forward_norm(hb, gamma, beta, EPS, drop, pooling=B.FAE_POOL_MEAN)
    x = pooled.clone()
    gy = torch.randn(y.shape, device="cuda", generator=gen)
    dgamma, dbeta = hp.backward_norm_sgd(hb, pooled, gy, lr, gamma, EPS, drop, pooling=B.FAE_POOL_MEAN)
    hp.sync()
    keep, scale = (None, 1.0) if p == 0 else R.keep_and_scale(S * 3, dim, p, 11, 5)
    ref = R.NormRef(x, gamma, beta, EPS, None if keep is None else keep.reshape(x.shape).cuda(), scale)
    R.assert_within(y, *ref.forward(torch.float32), "y")
    (gx, dg, db), (tx, tg, tb) = ref.backward(gy, torch.float32)
    R.assert_within(pooled, gx, tx, "gradient of the pooled rows")
    R.assert_within(dgamma, dg, tg, "dgamma")
    R.assert_within(dbeta, db, tb, "dbeta")
    for z in range(3):
        n = _lengths(hb, z).clamp(min=1)[:, None]  # an empty bag is zeros
        px, seg = _pool(w0[z].double(), hb, z)
        mag, _ = _pool(w0[z].double().abs(), hb, z)
        # six rows of a bag: five additions, then the length's reciprocal and a product with it
        assert bool(((x[:, z].double() - px / n).abs() <= 8 * R.U * mag / n).all())
        idx = hb.slots[z].long()

        def scatter(per_bag):
            return torch.zeros_like(w0[z], dtype=torch.float64).index_add_(0, idx, (per_bag / n)[seg])
        G, mag, tol = scatter(gx[:, z]), scatter(gx[:, z].abs()), scatter(tx[:, z])
        k = torch.zeros(rows[z], dtype=torch.float64, device="cuda").index_add_(0, idx, torch.ones(len(idx), dtype=torch.float64, device="cuda"))
        want = w0[z].double() - lr * G  # the sum pooling's bound, two roundings more for the bag's length
        R.assert_within(hp.hotW[z], want, lr * (tol + (k[:, None] + 5) * R.U * mag) + 2 * R.U * want.abs() + 1e-30, f"table {z}")


def test_mean_pooling_in_a_graph():
    """Replays move the tables as eager steps do."""
    rows, S, lr, dim = [500, 90, 40, 7], 200, 0.05, 20
    st = torch.cuda.Stream()
    hp = _tables(rows, dim, st.cuda_stream)
    hb = _batch(rows, S, 1, 5)
    gamma, beta = torch.randn((2, 4, dim), device="cuda")
    gy = torch.randn((S, 4, dim), device="cuda")
    hp.bwd_workspace(hb)
    torch.cuda.synchronize()
    start = [w.clone() for w in hp.hotW]

    def step():
        pooled, y = hp.forward_norm(hb, gamma, beta, EPS, pooling=B.FAE_POOL_MEAN)
        return (y, *hp.backward_norm_sgd(hb, pooled, gy, lr, gamma, EPS, pooling=B.FAE_POOL_MEAN))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        got = step()
    torch.cuda.synchronize()
    for w, s in zip(hp.hotW, start):
        w.copy_(s)
    seen = []
    for _ in range(4):
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        seen.append([t.clone() for t in (*got, *hp.hotW)])
    for w, s in zip(hp.hotW, start):
        w.copy_(s)
    torch.cuda.synchronize()
    for i in range(4):
        want = step()
        hp.sync()
        for a, b in zip(seen[i], (*want, *hp.hotW)):
            assert torch.equal(a, b)


def test_sum_pooling_is_the_default():
    rows, S, dim = [50, 9], 100, 16
    out = []
    for kw in ({}, {"pooling": B.FAE_POOL_SUM}):
        hp, hb = _tables(rows, dim), _batch(rows, S, 4, 6)
        pooled, y = hp.forward_norm(hb, **kw)
        hp.backward_norm_sgd(hb, pooled, y.clone(), 0.1, **kw)
        hp.sync()
        out.append(hp.hotW)
    for a, b in zip(*out):
        assert torch.equal(a, b)


def test_an_unknown_pooling_is_refused():
    rows, S, dim = [50, 9], 100, 16
    hp, hb = _tables(rows, dim), _batch(rows, S, 4, 6)
    before = [w.clone() for w in hp.hotW]
    pooled, y = hp.forward_norm(hb)
    with pytest.raises(B.FaeError):
        hp.forward_norm(hb, pooling=7)
    x = pooled.clone()
    with pytest.raises(ValueError):
        hp.backward_norm_sgd(hb, pooled, y.clone(), 0.1, pooling=7)
    hp.sync()
    for a, b in zip([*hp.hotW, pooled], [*before, x]):
        assert torch.equal(a, b)

"""A training step that ends in the softmax loss: pooled forward, layer norm, the loss over a hot table's rows, its gradients, clipping, and back
to the hot tables; eager and captured, against the same in 64 bits by automatic differentiation."""
import pytest
import torch

from paper_2103_00686_amd import binding as B
from paper_2103_00686_amd.hotpath import HotPath, HotBatch

pytestmark = pytest.mark.gpu


def _tables(rows, dim, stream=None):
    hp = HotPath(rows, dim, stream=stream)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    hp.n_hot = list(rows)
    hp.hotW = [torch.randn((r, dim), device="cuda", generator=gen) * 0.3 for r in rows]
    return hp


def _batch(rows, n, seed):
    gen = torch.Generator().manual_seed(seed)
    slots, offsets, lookups = [], [], []
    for z, r in enumerate(rows):
        lens = torch.ones(n, dtype=torch.int64) if z == 0 else torch.randint(0, 5, (n,), generator=gen)
        off = torch.cat([torch.zeros(1, dtype=torch.int64), lens.cumsum(0)])
        total = int(off[-1])
        slots.append(torch.randint(0, r, (total,), generator=gen).to(torch.int32).cuda())
        offsets.append(None if z == 0 else off.to(torch.int32).cuda())
        lookups.append(total)
    return HotBatch(n, slots, offsets, lookups)


def _step(hp, hb, gamma, beta, targets, g, lr, max_norm):
    """The first table's rows are the classes; the summary of a sample is the sum of its normalised rows."""
    pooled, y = hp.forward_norm(hb, gamma, beta)
    x = y.sum(1)
    loss, lse, mean = hp.softmax_loss(x, 0, targets, None, 0.5, keep=True)
    gx, gw = hp.softmax_loss_backward(x, 0, targets, lse, g, mean, None, 0.5)
    norm = hp.clip_gradients([gx, gw], max_norm)
    hp.hotW[0].sub_(gw, alpha=lr)
    dgamma, dbeta = hp.backward_norm_sgd(hb, pooled, gx[:, None].expand_as(y).contiguous(), lr, gamma)
    return loss, norm, gx, gw, dgamma, dbeta


def _reference(W, hb, gamma, beta, targets, g, max_norm):
    W = [w.double().clone().requires_grad_() for w in W]
    gamma, beta = gamma.double().requires_grad_(), beta.double().requires_grad_()
    pooled = []
    for z, (s, o) in enumerate(zip(hb.slots, hb.offsets)):
        if o is None:
            pooled.append(W[z][s.long()])
        else:
            owner = torch.repeat_interleave(torch.arange(hb.n_samples, device="cuda"), (o[1:] - o[:-1]).long())
            pooled.append(torch.zeros((hb.n_samples, W[z].shape[1]), dtype=torch.float64, device="cuda").index_add(0, owner, W[z][s.long()]))
    p = torch.stack(pooled, 1)
    mu = p.mean(2, keepdim=True)
    y = (p - mu) / ((p - mu).square().mean(2, keepdim=True) + float(torch.tensor(1e-5))).sqrt() * gamma + beta
    x = y.sum(1)
    xd, classes = x.detach().requires_grad_(), W[0].detach().clone().requires_grad_()
    z = 0.5 * xd @ classes.t()
    known = targets >= 0
    loss = (torch.logsumexp(z, 1) - z.gather(1, targets.clamp(min=0).long()[:, None])[:, 0]) * known
    gx, gw = torch.autograd.grad((loss * g.double()).sum(), [xd, classes])
    norm = (gx.square().sum() + gw.square().sum()).sqrt()
    f = min(1.0, max_norm / float(norm))
    grads = torch.autograd.grad((x * gx * f).sum(), [*W, gamma, beta])
    return loss.detach(), norm, gx * f, gw * f, grads


@pytest.mark.parametrize("max_norm", [0.05, 1e3])
def test_a_step(max_norm):
    rows, n, dim, lr = [700, 300, 50], 400, 64, 0.1
    hp = _tables(rows, dim)
    hb = _batch(rows, n, 2)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(4)
    gamma, beta = torch.rand((3, dim), device="cuda", generator=gen) + 0.5, torch.randn((3, dim), device="cuda", generator=gen) * 0.1
    targets = torch.randint(-100, rows[0], (n,), device="cuda", generator=gen).clamp(min=-1).to(torch.int32)
    g = torch.full((n,), 1.0 / n, device="cuda")
    W0 = [w.clone() for w in hp.hotW]
    rl, rn, rx, rw, grads = _reference(W0, hb, gamma, beta, targets, g, max_norm)
    loss, norm, gx, gw, dgamma, dbeta = _step(hp, hb, gamma, beta, targets, g, lr, max_norm)
    hp.sync()
    # Bounds: x sums three normalised rows (a few units of 2^-24 each); a score is off by some 400 units of its terms' sum, 64 terms of up to about
    # 2, so by 1e-4 at most; losses by twice that, gradients by 2e-4 of the terms, which are the largest gradients times a few
    assert float((loss - rl).abs().max()) <= 4e-4
    assert abs(float(norm) - float(rn)) <= 4e-4 * float(rn)
    for got, ref in ((gx, rx), (gw, rw), (dgamma, grads[-2]), (dbeta, grads[-1])):
        assert float((got.double() - ref).abs().max()) <= 1e-3 * float(ref.abs().max())
    W0[0] -= lr * gw
    for w, w0, gr in zip(hp.hotW, W0, grads):
        moved = w.double() - w0.double()
        assert float((moved + lr * gr).abs().max()) <= 1e-3 * lr * float(gr.abs().max()) + 2.0 ** -23


def test_a_captured_step():
    rows, n, dim, lr = [900, 40], 200, 32, 0.1
    st = torch.cuda.Stream()
    hp = _tables(rows, dim, st.cuda_stream)
    hb = _batch(rows, n, 5)
    gamma, beta = torch.ones((2, dim), device="cuda"), torch.zeros((2, dim), device="cuda")
    targets = torch.randint(0, rows[0], (n,), device="cuda").to(torch.int32)
    g = torch.full((n,), 1.0 / n, device="cuda")
    start = [w.clone() for w in hp.hotW]
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        want = [t.clone() for t in _step(hp, hb, gamma, beta, targets, g, lr, 0.1)] + [w.clone() for w in hp.hotW]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        got = _step(hp, hb, gamma, beta, targets, g, lr, 0.1)
    for _ in range(3):
        for w, s in zip(hp.hotW, start):
            w.copy_(s)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip([*got, *hp.hotW], want):
            assert torch.equal(a, b)
        eager = hp.softmax_loss(torch.randn((70, dim), device="cuda"), 0, torch.zeros(70, dtype=torch.int32, device="cuda"))
        hp.sync()
        assert bool(torch.isfinite(eager[0]).all())

"""The softmax loss's backward with the forward's losses beside the one without, eager and captured."""
import pytest
import torch

import loss_ref as R
from paper_2103_00686_amd import binding as B
from paper_2103_00686_amd.hotpath import HotPath

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def _make(seed, n, v, d, dtype):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    x, w, bias, g = (torch.randn(s, device="cuda", generator=gen) for s in ((n, d), (v, d), (v,), (n,)))
    t = torch.randint(-5, v, (n,), device="cuda", generator=gen).clamp(min=-1)
    g[::3] = 0.0
    return x.to(dtype), w.to(dtype), t.to(torch.int32), bias, g


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("n,v,d", [(1, 1, 1), (1, 70, 33), (130, 5, 40), (700, 3001, 100), (90, 400, 256)])
def test_both_forms_of_ordinary_rows(n, v, d, dtype):
    """Gradients of both signs and zeros, rows without a target: both are within the definition's bounds, and gx is the same."""
    hp = HotPath([1], 4)
    x, w, t, bias, g = _make(n + v, n, v, d, dtype)
    scale = d ** -0.5
    loss, lse, mean = hp.softmax_loss(x, w, t, bias, scale, keep=True)
    (_, _, _, _), (rw, dw, _, _), (rb, db) = R.LossRef(x, w, t, bias, scale).backward(g)
    plain = hp.softmax_loss_backward(x, w, t, lse, g, mean, bias, scale)
    kept = hp.softmax_loss_backward(x, w, t, lse, g, mean, bias, scale, loss=loss)
    hp.sync()
    for gx, gw, gb in (plain, kept):
        assert torch.equal(gx, plain[0])
        R.assert_within(gw, rw, dw, "gw")
        R.assert_within(gb, rb, db, "gbias")


def test_no_rows():
    hp = HotPath([1], 4)
    x, w, t, bias, g = _make(1, 0, 40, 16, F32)
    loss, lse, mean = hp.softmax_loss(x, w, t, bias, keep=True)
    gx, gw, gb = hp.softmax_loss_backward(x, w, t, lse, g, mean, bias, loss=loss)
    hp.sync()
    assert gx.shape == (0, 16) and not bool(gw.any()) and not bool(gb.any())


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_a_captured_step(dtype):
    """The same bits on every replay, with eager calls of another size between."""
    st = torch.cuda.Stream()
    hp = HotPath([1], 4, stream=st.cuda_stream)
    x, w, t, bias, g = _make(3, 400, 3000, 64, dtype)
    other = _make(4, 90, 700, 64, dtype)
    torch.cuda.synchronize()

    def step(x, w, t, bias, g):
        loss, lse, mean = hp.softmax_loss(x, w, t, bias, 0.2, keep=True)
        return [loss, lse, mean, *hp.softmax_loss_backward(x, w, t, lse, g, mean, bias, 0.2, loss=loss)]
    want, want_other = step(x, w, t, bias, g), step(*other)
    hp.sync()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        got = step(x, w, t, bias, g)
    for _ in range(3):
        for o in got:
            o.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        eager = step(*other)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got + eager, want + want_other))


def test_a_loss_of_another_size_or_type():
    hp = HotPath([1], 4)
    x, w, t, bias, g = _make(5, 30, 50, 8, F32)
    loss, lse, mean = hp.softmax_loss(x, w, t, keep=True)
    for bad, error in ((loss[:29], ValueError), (loss.double(), TypeError), (loss.cpu(), TypeError)):
        with pytest.raises(error):
            hp.softmax_loss_backward(x, w, t, lse, g, mean, loss=bad)
    gx = torch.empty_like(x)
    with pytest.raises(B.FaeError):  # an output on the losses
        hp.prepare_softmax_loss_backward(B.SoftmaxLoss(30, 50, 8, t), x, w, lse, g, gx, None, None, mean, gx.view(-1)[:30])()
    hp.sync()

"""The softmax loss's gradient of the classes over many rows, against the definition in 64 bits (loss_ref.py has the bounds)."""
import pytest
import torch

import loss_ref as R
from paper_2103_00686_amd.hotpath import HotPath

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def hp():
    return HotPath([1], 4)


def _rand(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return lambda *shape: torch.randn(shape, device="cuda", generator=gen)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_gradient_of_classes_over_more_rows_than_threads_of_a_grid(hp, dtype):
    """2^26 rows and more, of which one in 2^16 and the first and last have a target: each of these is found, and nothing beside them."""
    n, v = (1 << 26) + 1000, 3
    x = torch.ones((n, 1), dtype=dtype, device="cuda")
    at = torch.cat([torch.arange(0, n, 65_537, device="cuda"), torch.arange(n - 70, n, device="cuda")])
    rand = _rand(3)
    x[at, 0] = (2.0 ** (torch.arange(at.numel(), device="cuda") % 5 - 3) * (1 + rand(at.numel()).abs())).to(dtype)
    w = torch.tensor([[0.5], [1.0], [-1.0]], device="cuda").to(dtype)
    t = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    t[at] = (torch.arange(at.numel(), device="cuda") % v).to(torch.int32)
    g = torch.ones(n, device="cuda")
    g[at] = rand(at.numel())
    bias = torch.zeros(v, device="cuda")
    loss, lse, mean = hp.softmax_loss(x, w, t, bias, keep=True)
    gx, gw, gb = hp.softmax_loss_backward(x, w, t, lse, g, mean, bias)
    hp.sync()
    assert int((gx != 0).sum()) <= at.numel() and int((loss != 0).sum()) == at.numel()
    ref = R.LossRef(x[at], w, t[at], bias)
    (rx, dx, _, _), (rw, dw, _, _), (rb, db) = ref.backward(g[at])
    R.assert_within(loss[at], *ref.loss(), "loss")
    R.assert_within(gx[at], rx, dx, "gx")
    R.assert_within(gw, rw, dw, "gw")
    R.assert_within(gb, rb, db, "gbias")
    least = ref.backward(g[at])[1][2].min() / at.numel()
    assert float(dw.max()) < 4 * float(least) or dtype == BF16

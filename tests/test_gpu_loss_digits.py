"""Digits of the softmax loss and its gradients where they are small beside what stands next to them: rows that are sure of their target, tables whose
rows have much in common, gradients of very different sizes.  Every value is held to the sum of its own terms' absolute values, in 64 bits.

Bounds (u = 2^-24, h half a step of the type as a probability enters a product, fp32 16 u; LossRef has both, and e, a probability's relative error):
each term by e and h; the sum of K roundings of a term at random by 2 sqrt(K) + 16 units of the terms' sum in root mean square, and no
one of a million values by more than eight times that; of fp16 numbers, 2^-34 of the largest term for each term."""
import math

import pytest
import torch

import loss_ref as R
from paper_2103_00686_amd import binding as B
from paper_2103_00686_amd.hotpath import HotPath

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [F32, BF16, F16]


@pytest.fixture(scope="module")
def hp():
    return HotPath([1], 4)


def _rand(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return lambda *shape: torch.randn(shape, device="cuda", generator=gen)


def _at_random(terms):
    return 8 * R.U * (2 * terms ** 0.5 + 16)


def _others(ref):
    """The probabilities of all classes but the target, and their sum as a column."""
    p = ref.p * (1 - ref.hot)
    return p, p.sum(1)[:, None]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,v,d", [(150, 120_000, 64), (40, 100_000, 72), (300, 3000, 128), (3000, 6000, 64)])
def test_mean_of_rows_that_are_sure_of_their_target(hp, n, v, d, dtype):
    """The target 12 to 34 nats above all others: what is left to them is down to 1e-10, and their mean keeps its digits."""
    rand = _rand(n)
    w = 0.5 + 0.3 * rand(v, d)
    w[:, 0] = 0.0
    w[77, 0] = 1.0
    x = 0.1 * rand(n, d)
    x[:, 0] = torch.linspace(12.0, 34.0, n, device="cuda")
    x, w = x.to(dtype), w.to(dtype)
    t = torch.full((n,), 77, dtype=torch.int32, device="cuda")
    g = rand(n)
    loss, lse, mean = hp.softmax_loss(x, w, t, keep=True)
    gx = hp.softmax_loss_backward(x, w, t, lse, g, mean)[0]
    hp.sync()
    ref = R.LossRef(x, w, t)
    p, left = _others(ref)
    want = p @ ref.w - left * ref.w[77]
    size = p @ ref.w.abs() + left * ref.w[77].abs()
    err = (p * (ref.e + ref.h)) @ ref.w.abs() + (p * (ref.e + ref.h)).sum(1)[:, None] * ref.w[77].abs() + _at_random(ref.N * v / 16) * size
    if dtype != BF16:
        err += 2.0 ** -34 * p.max(1).values[:, None] * (ref.w.abs().sum(0) + v * ref.w[77].abs())
    assert float((err / size).max()) < 0.03  # the bound tells a lost class from a rounded one
    R.assert_within(mean, want, err, "mean")
    if dtype == F32:
        R.assert_within(gx, g.double()[:, None] * want, g.double().abs()[:, None] * (err + 4 * R.U * size), "gx")
    R.assert_within(loss, torch.log1p(left[:, 0] / (1 - left[:, 0])), left[:, 0] * (ref.dlse + ref.dz[:, 77] + ref.e.amax(1)), "loss")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,v", [(1, 300), (40, 3000), (200, 200_000)])
def test_rows_whose_target_is_beyond_all_powers(hp, n, v, dtype):
    """The target hundreds of nats above all others, and hundreds below."""
    rand = _rand(v)
    for top in (300.0, -300.0):
        x, w = (0.1 * rand(n, 32)).to(dtype), (0.5 * rand(v, 32)).to(dtype)
        bias = torch.zeros(v, device="cuda")
        bias[v // 2] = top
        t = torch.full((n,), v // 2, dtype=torch.int32, device="cuda")
        for keep in (False, True):
            loss, lse, *mean = hp.softmax_loss(x, w, t, bias, keep=keep)
            hp.sync()
            ref = R.LossRef(x, w, t, bias)
            R.assert_within(lse, ref.lse, ref.dlse, "lse")
            if top > 0:
                assert float(loss.max()) < 1e-35 and not bool((loss < 0).any())
                assert not keep or float(mean[0].abs().max()) < 1e-35
            else:
                R.assert_within(loss, *ref.loss(), "loss")
                if keep:
                    R.assert_within(mean[0], *ref.mean(), "mean")


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("n,v,d", [(300, 50, 64), (20, 400, 64), (500, 900, 200), (200, 300, 33)])
def test_what_all_classes_have_in_common_is_in_no_gradient(hp, n, v, d, dtype):
    """Rows of the table that differ by a few steps of their type around 1: the mean is held to their differences, not to the rows."""
    rand = _rand(v)
    step = torch.finfo(dtype).eps
    w = (1 + step * (rand(v, d) * 2).round().clamp(-6, 6)).to(dtype)
    x = rand(n, d).to(dtype)
    t = (4 + torch.arange(n, device="cuda") * 7 % (v - 4)).to(torch.int32)
    scale = 0.15 / (2 * step * math.sqrt(d))
    bias = 0.5 * rand(v)
    bias[:3] += 6.0  # most of what the target leaves goes to few classes: their roundings do not average out
    loss, lse, mean = hp.softmax_loss(x, w, t, bias, scale, keep=True)
    hp.sync()
    ref = R.LossRef(x, w, t, bias, scale)
    p, left = _others(ref)
    wt = ref.w[ref.t]
    want = p @ ref.w - left * wt
    middle = p @ ref.w / left  # P's roundings count by how far a row is from the others' mean, the scores' by how far from the target's
    apart = torch.stack([pe @ (ref.w - wr).abs() + ref.h * (pr @ (ref.w - mr).abs()) for pe, pr, wr, mr in zip(p * ref.e, p, wt, middle)])
    size = p @ ref.w.abs() + left * wt.abs()
    err = apart + _at_random(v / 16) * size
    if dtype == F16:
        err += 2.0 ** -34 * p.max(1).values[:, None] * (ref.w.abs().sum(0) + v * wt.abs())
    R.assert_within(mean, want, err, "mean")

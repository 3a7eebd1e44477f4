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


def _sure(n, v, least, most, dtype, seed):
    """Rows with targets of their own, `least` to `most` nats above all other classes."""
    rand = _rand(seed)
    d = n + 16
    x, w = torch.zeros((n, d), device="cuda"), torch.zeros((v, d), device="cuda")
    w[:, n:] = 0.5 + 0.3 * rand(v, 16)
    x[:, n:] = 0.3 * rand(n, 16)
    at = torch.arange(n, device="cuda")
    t = at * (v // n) + 3
    x[at, at] = torch.linspace(least, most, n, device="cuda")
    w[t, at] = 1.0
    return x.to(dtype), w.to(dtype), t.to(torch.int32), rand


def _gradients(ref, g):
    """(gw, gbias, bounds) with 1 - p of a target as the sum of the others' probabilities."""
    p, left = _others(ref)
    eo = (p * ref.e).sum(1)[:, None] / left + ref.dz.gather(1, ref.t[:, None]) + 16 * R.U  # of 1 - p
    g = g.double()[:, None]
    G, size = g * (p - ref.hot * left), g.abs() * (p + ref.hot * left)
    dG = g.abs() * (p * ref.e + ref.hot * left * eo)
    x, s = ref.x, abs(ref.scale)
    n = ref.n
    gw, tw = ref.scale * (G.t().contiguous() @ x), s * (size.t().contiguous() @ x.abs())
    dw = s * ((dG + size * ref.h).t().contiguous() @ x.abs()) + _at_random(ref.N * n / 16) * tw
    return gw, dw, tw, G.sum(0), dG.sum(0) + _at_random(n) * size.sum(0), size


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("v", [700, 40_000])
def test_gradient_of_a_target_that_is_sure(hp, v, dtype):
    """loss down to 1e-14: with the forward's loss, the target's gradient is that sum and no difference of two numbers next to 1."""
    n = 48
    x, w, t, rand = _sure(n, v, 14.0, 40.0, dtype, v)
    bias = 0.1 * rand(v)
    for g in (rand(n), rand(n).abs(), -rand(n).abs()):
        loss, lse, mean = hp.softmax_loss(x, w, t, bias, keep=True)
        gx, gw, gb = hp.softmax_loss_backward(x, w, t, lse, g, mean, bias, loss=loss)
        hp.sync()
        ref = R.LossRef(x, w, t, bias)
        rw, dw, tw, rb, db, size = _gradients(ref, g)
        live = size.sum(0) > 0
        assert float((db / size.sum(0))[live].max()) < 0.02
        R.assert_within(gb, rb, db, "gbias")
        if dtype != BF16:  # fp16 numbers of all probabilities beside the largest gradient
            dw = dw + 2.0 ** -38 * float(g.abs().max()) * ref.x.abs().sum(0)
        if dtype != F32:
            dw = dw + R.half_step(rw.abs() + dw, dtype)
        R.assert_within(gw, rw, dw, "gw")


@pytest.mark.parametrize("dtype", TYPES)
def test_gradient_of_a_target_without_the_loss(hp, dtype):
    """From lse alone 1 - p is a difference whose digits end at lse's, but it has no wrong sign."""
    n, v = 48, 700
    x, w, t, rand = _sure(n, v, 20.0, 60.0, dtype, 5)
    bias, g = 0.1 * rand(v), rand(n).abs()
    loss, lse, mean = hp.softmax_loss(x, w, t, bias, keep=True)
    gx, gw, gb = hp.softmax_loss_backward(x, w, t, lse, g, mean, bias)
    hp.sync()
    ref = R.LossRef(x, w, t, bias)
    p, left = _others(ref)
    from_others = (g.double()[:, None] * p).sum(0)
    assert bool((gb.double() <= from_others * 1.01)[t.long()].all())
    (_, _, _, _), (_, _, _, _), (rb, db) = ref.backward(g)
    R.assert_within(gb, rb, db, "gbias")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("width", [20, 64, 100, 200])
def test_classes_whose_gradients_are_small_beside_others(hp, width, dtype):
    """Seven groups of rows, each with its own classes, and gradients from 1 down to 2^-54: every class keeps the digits of its own sum (fp16:
    but for 2^-39 of the largest gradient for every row, far below half a step of 2^-24)."""
    rand = _rand(width)
    groups, per, classes = 7, 40, 900
    n, v = groups * per, groups * classes
    x, w = 0.2 * rand(n, width), 0.5 + 0.3 * rand(v, width)
    x[:, :groups], w[:, :groups] = 0.0, 0.0
    row, cls = torch.arange(n, device="cuda") // per, torch.arange(v, device="cuda") % groups
    x[torch.arange(n, device="cuda"), row] = 45.0
    w[torch.arange(v, device="cuda"), cls] = 1.0
    t = (torch.randint(0, classes, (n,), device="cuda") * groups + row).to(torch.int32)
    x, w = x.to(dtype), w.to(dtype)
    g = rand(n) * 2.0 ** (-9.0 * row)
    bias = 0.1 * rand(v)
    for b in (None, bias):
        loss, lse, mean = hp.softmax_loss(x, w, t, b, keep=True)
        gx, gw, *gb = hp.softmax_loss_backward(x, w, t, lse, g, mean, b, loss=loss)
        hp.sync()
        ref = R.LossRef(x, w, t, b)
        rw, dw, tw, rb, db, size = _gradients(ref, g)
        dw = dw + 2.0 ** -126 * ref.x.abs().sum(0)  # the power is 0 below fp32's smallest normal number: a gradient of 2^-54 times a probability of 2^-75
        if dtype == F32:
            dw = dw + 2.0 ** -34 * size.amax(0)[:, None] * ref.x.abs().sum(0) + ref.mx * size.sum(0)[:, None]
        if dtype == F16:
            dw = dw + 2.0 ** -39 * float(g.abs().max()) * ref.x.abs().sum(0)
        else:
            assert float((dw / tw).median()) < 0.02
        if dtype != F32:
            dw = dw + R.half_step(rw.abs() + dw, dtype)
        R.assert_within(gw, rw, dw, "gw")
        if b is not None:
            R.assert_within(gb[0], rb, db, "gbias")


def test_all_rows_sure_of_their_targets_in_fp32(hp):
    """Nothing but small gradients: a class that is nobody's target has what the rows leave to it, down to 1e-24."""
    n, v = 48, 2000
    for least, most in ((30.0, 34.0), (20.0, 60.0)):
        x, w, t, rand = _sure(n, v, least, most, F32, 9)
        g = rand(n)
        loss, lse, mean = hp.softmax_loss(x, w, t, keep=True)
        gx, gw = hp.softmax_loss_backward(x, w, t, lse, g, mean, loss=loss)
        hp.sync()
        ref = R.LossRef(x, w, t)
        rw, dw, tw, _, _, size = _gradients(ref, g)
        R.assert_within(gw, rw, dw + 2.0 ** -34 * size.amax(0)[:, None] * ref.x.abs().sum(0) + ref.mx * size.sum(0)[:, None], "gw")

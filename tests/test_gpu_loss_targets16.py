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


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("n,v,d", [(200, 3000, 64), (1000, 900, 200), (40, 200_000, 32), (3000, 500, 96)])
def test_targets_enter_the_classes_gradient_unrounded(hp, n, v, d, dtype):
    """gw of 16-bit types: what a row leaves to its target, most of a class's gradient, enters as two numbers; the others' are off by half a step of
    themselves, each, and gw by half a step at the end."""
    rand = _rand(n)
    x, w = rand(n, d).to(dtype), (0.3 * rand(v, d)).to(dtype)
    t = (torch.arange(n, device="cuda") * 7 % v).to(torch.int32)
    x[::2] = (x[::2].float() + 0.7 * w[t[::2].long()].float() * d ** 0.5).to(dtype)
    g = rand(n)
    scale = 2.0 / math.sqrt(d)
    loss, lse, mean = hp.softmax_loss(x, w, t, None, scale, keep=True)
    gx, gw = hp.softmax_loss_backward(x, w, t, lse, g, mean, None, scale, loss=loss)
    hp.sync()
    ref = R.LossRef(x, w, t, None, scale)
    p, left = _others(ref)
    eo = (p * ref.e).sum(1)[:, None] / left + ref.dz.gather(1, ref.t[:, None]) + 16 * R.U
    ga = g.double().abs()[:, None]
    terms = scale * ((ga * (p + ref.hot * left)).t().contiguous() @ ref.x.abs())
    want = scale * ((g.double()[:, None] * (p - ref.hot * left)).t().contiguous() @ ref.x)
    err = scale * ((ga * (p * (ref.e + ref.h) + ref.hot * left * (eo + ref.h ** 2))).t().contiguous() @ ref.x.abs()) + _at_random(2 * n / 16) * terms
    if dtype == F16:
        err += scale * 2.0 ** -39 * float(g.abs().max()) * ref.x.abs().sum(0)
    R.assert_within(gw, want, err + R.half_step(want.abs() + err, dtype), "gw")

"""Rows of equal values up to where their sum ends: what is left of the mean's rounding after two means, 2^-38 of the value.

A lane adds up to 16 equal values one after the other and teams join at most ten sums in pairs, so the first mean errs by fewer than
27 roundings and the mean of the deviations by as much of these: (27 * 2^-24)^2 < 2^-38."""
import pytest
import torch

from paper_2103_00686_amd.hotpath import HotPath

pytestmark = pytest.mark.gpu

EPS = 1e-5


@pytest.fixture(scope="module")
def hp():
    return HotPath([1], 4)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("width", [1, 3, 7, 64, 100, 257, 1000, 1030, 1664, 4099, 9001, 16384])
def test_equal_values(hp, width, dtype):
    top = 3.3e38 / width
    v = torch.tensor([s * m * top * 10.0 ** -e for e in range(0, 38, 2) for m in (1.0, 0.7310585, 0.3333333) for s in (1, -1)], device="cuda")
    x = v[:, None].expand(-1, width).to(dtype).contiguous()
    y = hp.layer_norm(x, eps=EPS)
    gx, dgamma, dbeta = hp.layer_norm_backward(x, torch.zeros_like(x), eps=EPS)
    hp.sync()
    most = x.double().abs() * 2.0 ** -38 / EPS ** 0.5 * 1.01  # the results' own rounding
    assert bool((y.double().abs() <= most).all())
    assert not bool(gx.any()) and not bool(dgamma.any()) and not bool(dbeta.any())


def test_zeros(hp):
    for eps in (1e-5, 1.1754944e-38, 1e-40):  # the last is below the normal range
        for width in (16, 100, 2000):
            x = torch.zeros((9, width), device="cuda")
            y = hp.layer_norm(x, eps=eps)
            gx, dg, db = hp.layer_norm_backward(x, torch.zeros_like(x), eps=eps)
            hp.sync()
            assert not bool(y.any()) and not bool(gx.any()) and not bool(dg.any()) and not bool(db.any())

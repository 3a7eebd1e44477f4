"""Clipping where the norm, or its limit, is infinite."""
import math

import pytest
import torch

from paper_2103_00686_amd.hotpath import HotPath

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_an_infinite_gradient_under_any_limit(dtype):
    """Without a limit (infinite max_norm) an infinite norm says the same as with one: finite values 0, infinite ones NaN."""
    hp = HotPath([1], 4)
    for max_norm in (1.0, math.inf):
        g = torch.ones(5000, device="cuda").to(dtype)
        g[4711] = -math.inf
        norm = hp.clip_gradients([g], max_norm)
        hp.sync()
        assert float(norm) == math.inf and math.isnan(float(g[4711]))
        g[4711] = 0
        assert not bool(g.any())


def test_a_norm_beyond_fp32_without_a_limit():
    """... but finite gradients whose norm fp32 cannot hold are left as they are."""
    hp = HotPath([1], 4)
    g = torch.full((5000,), 3e38, device="cuda")
    norm = hp.clip_gradients([g], math.inf)
    hp.sync()
    assert float(norm) == math.inf and bool((g == 3e38).all())

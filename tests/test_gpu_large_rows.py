"""Layer norm and dropout of as many rows as their headers allow: more threads than one grid holds."""
import numpy as np
import pytest
import torch

import rows_ref as R
from paper_2103_00686_amd import binding as B
from paper_2103_00686_amd.hotpath import HotPath

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16
PIECE = 1 << 28  # values looked at together


@pytest.fixture(scope="module")
def hp():
    yield HotPath([1], 4)
    torch.cuda.empty_cache()


def _numbers(rows, cols, seed, offset):
    """The generator's numbers of single values (64-bit integer arithmetic on the host)."""
    m, sh = np.uint64(0xFFFFFFFF), np.uint64(32)
    cols = np.asarray(cols, dtype=np.uint64)
    c0, c1 = cols >> np.uint64(3), np.asarray(rows, dtype=np.uint64)
    c2, c3 = np.full_like(c0, offset & 0xFFFFFFFF), np.full_like(c0, offset >> 32)
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32
    for _ in range(10):
        a, b = c0 * np.uint64(0xD2511F53), c2 * np.uint64(0xCD9E8D57)
        c0, c1, c2, c3 = (b >> sh) ^ c1 ^ np.uint64(k0), b & m, (a >> sh) ^ c3 ^ np.uint64(k1), a & m
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    words = np.stack([c0, c1, c2, c3], 1).astype(np.uint32).view(np.uint16)
    return words[np.arange(len(cols)), (cols & np.uint64(7)).astype(np.int64)].astype(np.int64)


def test_numbers_of_single_values():
    rows, cols = (v.ravel() for v in np.meshgrid(np.arange(50), np.arange(21), indexing="ij"))
    assert np.array_equal(_numbers(rows, cols, 77, 5).reshape(50, 21), R.philox_numbers(50, 21, 77, 5))


@pytest.mark.parametrize("backward", [False, True])
def test_dropout_of_the_most_rows(hp, backward):
    """2^32 - 1 rows of one value, a thread each: all are taken, once, with the mask of their own row."""
    n, seed, offset = (1 << 32) - 1, 0xFEDCBA9876543210, (1 << 40) + 3
    x = torch.ones((n, 1), dtype=F16, device="cuda")
    drop = B.Drop(0.5, seed, offset)
    (hp.dropout_backward if backward else hp.dropout)(x, drop, out=x)
    hp.sync()
    kept = 0
    for i in range(0, n, PIECE):
        v = x[i:i + PIECE]
        k = int((v == 2).sum())
        assert k + int((v == 0).sum()) == v.numel()
        kept += k
    assert abs(kept - n / 2) < 6 * (n / 4) ** 0.5
    rng = np.random.default_rng(1)
    edges = [0, 1 << 24, 1 << 31, n]  # where launches, grids and 32-bit numbers end
    rows = np.unique(np.concatenate([rng.integers(0, n, 20000)] + [np.clip(np.arange(e - 600, e + 600), 0, n - 1) for e in edges]))
    got = x[torch.from_numpy(rows).cuda(), 0].float().cpu().numpy()
    assert np.array_equal(got, np.where(_numbers(rows, 0 * rows, seed, offset) < 32768, 0.0, 2.0))


def test_dropout_of_long_rows_past_a_grid(hp):
    """Nine rows of 2^31 - 8 values: more than 2^31 groups of eight."""
    n, width, seed = 9, (1 << 31) - 8, 5
    x = torch.full((n, width), 3.0, dtype=F16, device="cuda")
    hp.dropout(x, B.Drop(0.25, seed, 9), out=x)
    hp.sync()
    four = 4.0  # 3 * (4 / 3 in fp32), rounded to fp16
    rng = np.random.default_rng(2)
    for r in range(n):
        kept = 0
        for i in range(0, width, PIECE):
            v = x[r, i:i + PIECE]
            k = int((v == four).sum())
            assert k + int((v == 0).sum()) == v.numel()
            kept += k
        assert abs(kept - 0.75 * width) < 6 * (width * 0.1875) ** 0.5
        cols = np.unique(np.concatenate([rng.integers(0, width, 4000), np.arange(100), width - 1 - np.arange(100)]))
        got = x[r][torch.from_numpy(cols).cuda()].float().cpu().numpy()
        assert np.array_equal(got, np.where(_numbers(np.full(len(cols), r), cols, seed, 9) < 16384, 0.0, four))


# More workgroups than one grid takes: teams of two lanes (four rows each at a time), of two waves with one row at a time, several parts
# whose number does not divide the teams.
@pytest.mark.parametrize("dtype,rows,parts,width,p", [(BF16, (1 << 30) + 777, 1, 2, 0.0), (BF16, (1 << 31) - 1, 1, 1, 0.5), (BF16, (1 << 30) // 3 + 5000, 3, 3, 0.25),
                                                      (BF16, (1 << 25) + 99, 1, 264, 0.0), (torch.float32, (1 << 21) + 1234, 1, 1028, 0.25)])
def test_layer_norm_past_a_grid(hp, dtype, rows, parts, width, p):
    """Every row is what a call on a few rows gives, and is dropped as dropout alone drops it."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(width)
    x = torch.empty((rows, parts * width), dtype=dtype, device="cuda")
    x.uniform_(-3, 3, generator=gen)
    x = x.view(rows, parts, width)
    gamma, beta = (torch.randn((parts, width), device="cuda", generator=gen) for _ in range(2))
    beta += torch.where(beta < 0, -40.0, 40.0)  # no kept value is zero: |gamma h| < 40, as |h| < 2 for uniform values
    drop = B.Drop(p, 21, 4) if p > 0 else None
    y = torch.full_like(x, float("nan"))
    hp.layer_norm(x, gamma, beta, drop=drop, out=y)
    hp.sync()
    flat = y.view(-1)
    assert not any(bool(flat[i:i + PIECE].isnan().any()) for i in range(0, flat.numel(), PIECE))
    if drop is not None:
        mask = hp.dropout(torch.ones_like(x), drop)
        hp.sync()
        mask = mask.view(-1)
        for i in range(0, flat.numel(), PIECE):
            assert torch.equal(flat[i:i + PIECE] != 0, mask[i:i + PIECE] != 0)
    step = max(1, PIECE // (parts * width))
    scale = torch.tensor(65536 / (65536 - round(65536 * p)), device="cuda")  # dropout's factor is in the weights
    for i in range(0, rows, step):
        part = x[i:i + step]
        want = hp.layer_norm(part, gamma * scale, beta * scale)
        hp.sync()
        got = y[i:i + step]
        assert torch.equal(got, want) if drop is None else bool(((got == want) | (got == 0)).all())


@pytest.mark.parametrize("parts", [1, 3])
def test_backward_of_the_most_rows(hp, parts):
    """n_rows * n_parts as near to 2^31 as it goes; gradients of zero but for a few samples at the end, so that the sums are theirs."""
    rows, width, last = ((1 << 31) - 1) // parts, 2, 700
    gen = torch.Generator(device="cuda")
    gen.manual_seed(parts)
    x = torch.empty((rows, parts, width), dtype=BF16, device="cuda").uniform_(-3, 3, generator=gen)
    gy = torch.zeros_like(x)
    gy[-last:] = torch.randn((last, parts, width), device="cuda", generator=gen).to(BF16)
    gamma = torch.randn((parts, width), device="cuda", generator=gen)
    gx = torch.full_like(x, float("nan"))
    _, dgamma, dbeta = hp.layer_norm_backward(x, gy, gamma, out=gx)
    hp.sync()
    (rx, rg, rb), (tx, tg, tb) = R.NormRef(x[-last:], gamma, None, 1e-5).backward(gy[-last:], BF16)
    R.assert_within(gx[-last:], rx, tx, "gx")
    R.assert_within(dgamma.reshape(parts, width), rg, tg, "dgamma")
    R.assert_within(dbeta.reshape(parts, width), rb, tb, "dbeta")
    flat = gx[:-last].reshape(-1)
    assert not any(bool((flat[i:i + PIECE] != 0).any()) for i in range(0, flat.numel(), PIECE))


def test_dropout_of_samples_with_gaps_past_a_grid(hp):
    """Three parts and a gap in every sample: launches start at a sample, rows count on."""
    n, parts = (1 << 31) // 3 + 70_001, 3
    flat = torch.ones((n, 4), dtype=F16, device="cuda")
    x = flat[:, :3].unflatten(1, (parts, 1))
    hp.dropout(x, B.Drop(0.5, 3, 8), out=x)
    hp.sync()
    step = PIECE // 4
    for i in range(0, n, step):
        v = flat[i:i + step]
        assert bool((v[:, 3] == 1).all()) and bool(((v[:, :3] == 0) | (v[:, :3] == 2)).all())
    rng = np.random.default_rng(3)
    border = (1 << 31) // 3
    samples = np.unique(np.concatenate([rng.integers(0, n, 8000), np.arange(300), border - 150 + np.arange(300), n - 1 - np.arange(300)]))
    got = flat[torch.from_numpy(samples).cuda(), :3].float().cpu().numpy().ravel()
    rows = (samples[:, None] * 3 + np.arange(3)).ravel()
    assert np.array_equal(got, np.where(_numbers(rows, 0 * rows, 3, 8) < 32768, 0.0, 2.0))

"""Dropout against its definition: the mask bit for bit from the generator on the host, kept values with the one rounding of
their product and the one of their type."""
import numpy as np
import pytest
import torch

import rows_ref as R
from paper_2103_00686_amd import binding as B
from paper_2103_00686_amd.hotpath import HotPath

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [(F32, F32), (F32, BF16), (F32, F16), (BF16, F32), (F16, F32), (BF16, BF16), (F16, F16)]
SEED = 0xFEDCBA9876543210


@pytest.fixture(scope="module")
def hp():
    return HotPath([1], 4)


def _want(x, p, seed, offset, dtype):
    """Each kept value times fp32's factor, rounded to fp32 and to its type: exact, there is nothing else to round."""
    rows = x.shape[0] * (x.shape[1] if x.dim() == 3 else 1)
    keep, scale = R.keep_and_scale(rows, x.shape[-1], p, seed, offset)
    return torch.where(keep.reshape(x.shape).cuda(), x.float() * float(np.float32(scale)), 0.0).to(dtype)


def _gapped(x, pad, lead):
    flat = torch.full((lead + x.shape[0] * (x[0].numel() + pad),), float("nan"), dtype=x.dtype, device="cuda")
    v = flat[lead:].view(x.shape[0], -1)[:, :x[0].numel()].unflatten(1, x.shape[1:])
    v.copy_(x)
    return flat, v


@pytest.mark.parametrize("tx,ty", TYPES)
@pytest.mark.parametrize("shape", [(1, 1), (1, 7), (3, 8), (5, 9), (7, 16), (64, 50), (33, 3, 20), (17, 26, 64), (100, 100), (11, 1031), (2, 5, 333), (4, 16384), (1, 70001)])
def test_shapes_and_types(hp, shape, tx, ty):
    x = torch.randn(shape, device="cuda").to(tx)
    drop = B.Drop(0.3, SEED, 5)
    y = hp.dropout(x, drop, ty)
    hp.sync()
    assert torch.equal(y, _want(x, 0.3, SEED, 5, ty))
    gx = hp.dropout_backward(x, drop, ty)
    hp.sync()
    assert torch.equal(gx, y)  # the gradient goes through the same mask


@pytest.mark.parametrize("tx,ty", TYPES)
@pytest.mark.parametrize("shape,pad,lead", [((9, 64), 3, 1), ((5, 3, 50), 7, 3), ((3, 1000), 8, 5), ((6, 24), 8, 8)])
def test_gaps(hp, shape, pad, lead, tx, ty):
    _, x = _gapped(torch.randn(shape, device="cuda").to(tx), pad, lead)
    flat, y = _gapped(torch.zeros(shape, dtype=ty, device="cuda"), pad, lead)
    hp.dropout(x, B.Drop(0.5, SEED, 1 << 35), out=y)
    hp.sync()
    assert torch.equal(y, _want(x, 0.5, SEED, 1 << 35, ty))
    assert int(torch.isnan(flat).sum()) == flat.numel() - y.numel()


@pytest.mark.parametrize("p", [0.0, 1.0, 2.0 ** -16, 1 - 2.0 ** -16, 0.1, 0.5, 0.9])
def test_shares(hp, p):
    x = torch.randn((40, 264), device="cuda")
    y = hp.dropout(x, B.Drop(p, 7, 0))
    hp.sync()
    assert torch.equal(y, _want(x, p, 7, 0, F32))
    assert p != 0.0 or torch.equal(y, x)
    assert p != 1.0 or not bool(y.any())


def test_how_often_and_how_far_apart(hp):
    """16 M values: the dropped share is p's within six standard deviations, and neighbours, rows and successive offsets do not
    follow each other (correlations of independent draws have the deviation 1 / sqrt(n))."""
    x = torch.ones((16384, 1024), device="cuda")
    p = 0.1
    a, b = (hp.dropout(x, B.Drop(p, 123, o)) > 0 for o in (0, 1))
    c = hp.dropout(x, B.Drop(p, 124, 0)) > 0
    hp.sync()
    n = x.numel()
    t = round(p * 65536) / 65536
    for m in (a, b, c):
        assert abs(1 - float(m.double().mean()) - t) < 6 * (t * (1 - t) / n) ** 0.5
    z = [(m.double() - (1 - t)) / (t * (1 - t)) ** 0.5 for m in (a, b, c)]
    pairs = [(z[0], z[1]), (z[0], z[2]), (z[0][:, 1:], z[0][:, :-1]), (z[0][:, 8:], z[0][:, :-8]), (z[0][1:], z[0][:-1])]
    for u, v in pairs:
        assert abs(float((u * v).mean())) < 6 / n ** 0.5


def test_dropped_values_are_zero_whatever_they_were(hp):
    x = torch.full((50, 96), float("nan"), device="cuda")
    keep = R.keep_and_scale(50, 96, 0.4, 3, 2)[0].cuda()
    x[keep] = 1.0
    y = hp.dropout(x, B.Drop(0.4, 3, 2))
    hp.sync()
    assert torch.equal(y != 0, keep) and not bool(torch.isnan(y).any())


def test_in_place_and_side_by_side(hp):
    x = torch.randn((50, 96), device="cuda")
    drop = B.Drop(0.4, 3, 2)
    want = hp.dropout(x, drop)
    both = torch.zeros((50, 200), device="cuda")
    both[:, :96] = x
    hp.dropout(both[:, :96], drop, out=both[:, 100:196])
    hp.dropout(x, drop, out=x)
    hp.sync()
    assert torch.equal(x, want) and torch.equal(both[:, 100:196], want)


def test_the_norm_has_the_same_mask(hp):
    """What layer norm drops is what dropout alone drops of rows of the same shape."""
    x = torch.randn((37, 5, 100), device="cuda")
    drop = B.Drop(0.35, 17, 1 << 33)
    beta = torch.full((5, 100), 1e4, device="cuda")
    y = hp.layer_norm(x, None, beta, drop=drop)
    d = hp.dropout(torch.ones_like(x), drop)
    hp.sync()
    assert torch.equal(y != 0, d != 0)


def test_captured_with_the_offset_on_the_device(hp):
    st = torch.cuda.Stream()
    hp = HotPath([1], 4, stream=st.cuda_stream)
    x, y = torch.randn((300, 130), device="cuda"), torch.empty((300, 130), device="cuda")
    counter = torch.zeros(1, dtype=torch.int64, device="cuda")
    call = hp.prepare_dropout(B.Drop(0.2, 5, 100, counter), x, y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        call()
    for step in (0, 1, -100, 1 << 40):  # the sum is modulo 2^64
        counter.fill_(step)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, _want(x, 0.2, 5, (100 + step) % (1 << 64), F32))


def test_offsets_past_32_bits(hp):
    n, stride = 65539, 65576
    x = torch.empty(n * stride, dtype=F16, device="cuda").view(n, stride)[:, 3:19]
    x.copy_(torch.randn((n, 16), device="cuda"))
    drop = B.Drop(0.5, 1, 1)
    a, b = hp.dropout(x, drop), hp.dropout(x.contiguous(), drop)
    hp.sync()
    assert torch.equal(a, b)


def test_no_rows(hp):
    assert hp.dropout(torch.empty((0, 5), device="cuda"), B.Drop(0.5, 1)).numel() == 0
    hp.sync()

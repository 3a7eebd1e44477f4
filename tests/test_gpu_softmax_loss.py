"""Softmax cross entropy over a table's rows and its gradients, against the definition in 64 bits (loss_ref.py has the bounds)."""
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


def _buf(n, width, dtype, pad, lead):
    """[n, width] with `pad` values behind every row and `lead` in front of the first, all NaN."""
    flat = torch.full((lead + n * (width + pad),), float("nan"), dtype=dtype, device="cuda")
    return flat, flat[lead:].view(n, width + pad)[:, :width]


def _make(seed, n, v, d, dtype, bias=False, pad=0, lead=0, size=1.0, cold=0.1):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def rand(*shape):
        return torch.randn(shape, device="cuda", generator=gen)
    x, w = _buf(n, d, dtype, pad, lead)[1], _buf(v, d, dtype, pad, lead)[1]
    w.copy_(rand(v, d) * size)
    t = torch.randint(0, v, (n,), device="cuda", generator=gen)
    x.copy_(rand(n, d) + 0.5 * w[t].float())
    t[torch.rand(n, device="cuda", generator=gen) < cold] = -1
    return x, w, t.to(torch.int32), rand(v) if bias else None, rand(n)


def _check(hp, x, w, t, bias, g, scale, pad=0, lead=0, with_mean=True, ref=None):
    n, d = x.shape
    v = w.shape[0]
    what = B.SoftmaxLoss(n, v, d, t, bias, scale, x.dtype)
    loss, lse = torch.empty((2, n), device="cuda")
    mean = torch.empty((n, d), device="cuda") if with_mean else None
    (xflat, gx), (wflat, gw) = _buf(n, d, x.dtype, pad, lead), _buf(v, d, x.dtype, pad, lead)
    gb = torch.empty(v, device="cuda") if bias is not None else None
    x0, w0 = x.clone(), w.clone()
    hp.prepare_softmax_loss(what, x, w, loss, lse, mean)()
    hp.prepare_softmax_loss_backward(what, x, w, lse, g, gx, gw, gb, mean)()
    hp.sync()
    assert torch.equal(torch.nan_to_num(x), torch.nan_to_num(x0)) and torch.equal(w, w0)
    ref = ref or R.LossRef(x, w, t, bias, scale)
    R.assert_within(lse, ref.lse, ref.dlse, "lse")
    R.assert_within(loss, *ref.loss(), "loss")
    if with_mean:
        live = ~ref.empty
        m, dm = ref.mean()
        R.assert_within(mean[live], m[live], dm[live], "mean")
    (rx, dx, tx, kx), (rw, dw, tw, kw), (rb, db) = ref.backward(g)
    R.assert_within(gx, rx, dx, "gx")
    R.assert_within(gw, rw, dw, "gw")
    if gb is not None:
        R.assert_within(gb, rb, db, "gbias")
    if x.dtype == F32 and ref.dlse.numel() and float(ref.dlse.max()) < 1e-3:
        spread = (ref.p * R.U * (2 * (6 * d / 16) ** 0.5 + 16) * (ref.x.abs() @ ref.w.abs().t().contiguous()) * abs(ref.scale)).sum(1)
        more = 1 + float(spread.mean() / R.U) / 8  # what the scores' own roundings do to a probability
        R.assert_rms(gx, rx, tx * more, kx, "gx")
        R.assert_rms(gw, rw, tw * more, kw, "gw")
    for flat, out in ((xflat, gx), (wflat, gw)):  # what lies in front of, behind and between the rows was left as it was
        assert int(torch.isnan(flat).sum()) == flat.numel() - out.numel()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("width", [1, 2, 3, 5, 7, 8, 9, 15, 16, 17, 31, 32, 33, 48, 63, 64, 65, 96, 97, 100, 127, 128, 129, 160, 191, 192, 193, 200, 255, 256])
def test_widths(hp, width, dtype):
    odd = width % 3
    x, w, t, bias, g = _make(width, 70, 531, width, dtype, bias=width % 2 == 0, pad=(0, 8, 5)[odd], lead=odd)
    _check(hp, x, w, t, bias, g, 1.5 / math.sqrt(width), (0, 8, 5)[odd], odd, with_mean=width % 4 != 3)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,v", [(1, 1), (1, 2), (2, 1), (1, 63), (1, 64), (3, 65), (31, 127), (32, 128), (33, 129), (127, 1000), (128, 31), (129, 32),
                                 (500, 33), (1, 20_011), (7, 4099), (260, 5003), (2000, 7), (5001, 130), (1000, 1)])
def test_sizes(hp, n, v, dtype):
    x, w, t, bias, g = _make(n * 31 + v, n, v, 40, dtype, bias=v % 2 == 1)
    _check(hp, x, w, t, bias, g, 0.2)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,v,d", [(130, 70_001, 64), (9000, 300, 64), (700, 3000, 256)])
def test_many_parts(hp, n, v, d, dtype):
    x, w, t, bias, g = _make(n + v, n, v, d, dtype, bias=True)
    _check(hp, x, w, t, bias, g / n, 1.0 / math.sqrt(d))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("scale", [-0.3, 0.0, 3.0, 20.0])
def test_scales(hp, scale, dtype):
    """Negative, none, and confident rows (the largest probability of most is 1 to many digits)."""
    x, w, t, bias, g = _make(5, 200, 700, 64, dtype, bias=True, size=0.3)
    _check(hp, x, w, t, bias, g, scale)


@pytest.mark.parametrize("dtype", TYPES)
def test_scores_that_rise_and_fall(hp, dtype):
    """The running maximum moves in every tile, or only in the first; scores of hundreds."""
    for way in (1, -1):
        x, w, t, _, g = _make(8, 150, 2000, 32, dtype)
        bias = torch.linspace(-300.0, 300.0, 2000, device="cuda") * way
        _check(hp, x, w, t, bias, g, 0.1)


@pytest.mark.parametrize("dtype", TYPES)
def test_classes_that_are_not_offered(hp, dtype):
    x, w, t, bias, g = _make(3, 100, 600, 48, dtype, bias=True)
    bias[torch.rand(600, device="cuda") < 0.5] = -math.inf
    bias[:70] = -math.inf  # the first tile has none
    bias[t.clamp(min=0).long()[:50]] = 0.5
    assert bool(torch.isinf(bias[t[50:].clamp(min=0).long()]).any())  # some targets are not offered: loss +inf, gradients finite
    _check(hp, x, w, t, bias, g, 0.2)


@pytest.mark.parametrize("dtype", TYPES)
def test_no_class_is_offered(hp, dtype):
    x, w, t, bias, g = _make(3, 20, 200, 48, dtype, bias=True)
    bias.fill_(-math.inf)
    loss, lse, mean = hp.softmax_loss(x, w, t, bias, 0.3, keep=True)
    gx, gw, gb = hp.softmax_loss_backward(x, w, t, lse, g, mean, bias, 0.3)
    hp.sync()
    assert bool((lse == -math.inf).all())
    for out in (loss, mean, gx, gw, gb):
        assert not bool(out.any())


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_without_a_target(hp, dtype):
    """They may hold anything: the others' gradients do not see it, their own are 0."""
    x, w, t, bias, g = _make(4, 200, 300, 64, dtype, bias=True, cold=0.4)
    want = [o.clone() for o in hp.softmax_loss_backward(x, w, t, hp.softmax_loss(x, w, t, bias, 0.2)[1], g, None, bias, 0.2)]
    cold = t < 0
    x[cold] = float("nan")
    g[cold] = float("inf")
    loss, lse = hp.softmax_loss(x, w, t, bias, 0.2)
    gx, gw, gb = hp.softmax_loss_backward(x, w, t, lse, g, None, bias, 0.2)
    hp.sync()
    assert not bool(loss[cold].any()) and not bool(gx[cold].any())
    for a, b in zip((gx, gw, gb), want):
        assert torch.equal(a, b)


def test_targets_of_64_bits_and_out_of_range(hp):
    x, w, t, bias, g = _make(6, 300, 500, 32, F32)
    want = hp.softmax_loss(x, w, t)
    got = hp.softmax_loss(x, w, t.long())
    hp.sync()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    for wrong in (500, 2 ** 31 - 1, 2 ** 31, 2 ** 33 + 5, 2 ** 62):
        bad = t.long()
        bad[7] = wrong
        off = t.long()
        off[7] = -1
        loss, lse, mean = hp.softmax_loss(x, w, bad, keep=True)
        with pytest.raises(B.FaeError) as e:
            hp.sync()
        assert e.value.code == B.FAE_ERANGE
        gx, gw = hp.softmax_loss_backward(x, w, bad, lse, g, mean)
        with pytest.raises(B.FaeError):
            hp.sync()
        l2, e2, m2 = hp.softmax_loss(x, w, off, keep=True)
        for a, b in zip((loss, lse, mean, gx, gw), (l2, e2, m2, *hp.softmax_loss_backward(x, w, off, e2, g, m2))):
            assert torch.equal(a, b)
        hp.sync()
    hp.softmax_loss(x, w, torch.full((300,), -2 ** 40, dtype=torch.int64, device="cuda"))
    hp.sync()


@pytest.mark.parametrize("dtype", TYPES)
def test_no_rows(hp, dtype):
    w = torch.randn((70, 30), device="cuda").to(dtype)
    x, t = torch.empty((0, 30), dtype=dtype, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda")
    bias = torch.zeros(70, device="cuda")
    loss, lse, mean = hp.softmax_loss(x, w, t, bias, keep=True)
    gx, gw, gb = hp.softmax_loss_backward(x, w, t, lse, loss, mean, bias)
    hp.sync()
    assert loss.numel() == 0 and gx.shape == (0, 30) and not bool(gw.any()) and not bool(gb.any())


def test_parts_of_the_outputs(hp):
    """Each output alone is what it is beside the others, without mean as with it."""
    x, w, t, bias, g = _make(9, 140, 900, 72, F32, bias=True)
    what = B.SoftmaxLoss(140, 900, 72, t, bias, 0.2, F32)
    loss, lse, mean = hp.softmax_loss(x, w, t, bias, 0.2, keep=True)
    one = torch.empty((2, 140), device="cuda")
    hp.prepare_softmax_loss(what, x, w, one[0], None)()
    hp.prepare_softmax_loss(what, x, w, None, one[1])()
    gx, gw, gb = hp.softmax_loss_backward(x, w, t, lse, g, mean, bias, 0.2)
    x1, w1, b1 = torch.empty_like(gx), torch.empty_like(gw), torch.empty_like(gb)
    hp.prepare_softmax_loss_backward(what, x, w, lse, g, x1, None)()
    hp.prepare_softmax_loss_backward(what, x, w, lse, g, None, w1)()
    hp.prepare_softmax_loss_backward(what, x, w, lse, g, None, None, b1)()
    hp.prepare_softmax_loss_backward(what, x, w, lse, g, None, None)()
    hp.sync()
    for a, b in ((one[0], loss), (one[1], lse), (x1, gx), (w1, gw), (b1, gb)):
        assert torch.allclose(a, b, rtol=1e-5, atol=1e-6)
    assert torch.equal(w1, gw) and torch.equal(b1, gb)


def test_values_that_are_not_finite(hp):
    """A row of x with NaN spoils its own loss and gradient and the classes', no other row's."""
    x, w, t, _, g = _make(11, 90, 300, 32, F32, cold=0.0)
    loss0, lse0, mean0 = hp.softmax_loss(x, w, t, None, 0.3, keep=True)
    x[5, 3] = float("nan")
    loss, lse, mean = hp.softmax_loss(x, w, t, None, 0.3, keep=True)
    gx, gw = hp.softmax_loss_backward(x, w, t, lse, g, mean, None, 0.3)
    hp.sync()
    rest = torch.arange(90, device="cuda") != 5
    assert torch.equal(loss[rest], loss0[rest]) and torch.equal(mean[rest], mean0[rest]) and not bool(torch.isnan(gx[rest]).any())
    assert math.isnan(float(loss[5])) and math.isnan(float(lse[5])) and bool(torch.isnan(gx[5]).all()) and bool(torch.isnan(gw).any())


def test_against_differences(hp):
    """The loss along a direction in x and w: (f(h) - f(-h)) / 2h is the gradient's part up to h^2 / 6 of the third derivative and the rounding
    of the two sums of losses, which 64 bits of the definition give without one."""
    x, w, t, bias, g = _make(12, 60, 200, 24, F32, bias=True)
    loss, lse, mean = hp.softmax_loss(x, w, t, bias, 0.4, keep=True)
    gx, gw, gb = hp.softmax_loss_backward(x, w, t, lse, g, mean, bias, 0.4)
    hp.sync()
    dx, dw, db = torch.randn_like(x).double(), torch.randn_like(w).double(), torch.randn_like(bias).double()

    def f(h):
        z = float(torch.tensor(0.4)) * ((x.double() + h * dx) @ (w.double() + h * dw).t().contiguous()) + bias.double() + h * db
        at = z.gather(1, t.clamp(min=0).long()[:, None])[:, 0]
        return float((torch.where(t >= 0, torch.logsumexp(z, 1) - at, torch.zeros_like(at)) * g.double()).sum())
    h = 1e-4
    d1, d2 = (f(h) - f(-h)) / (2 * h), (f(2 * h) - f(-2 * h)) / (4 * h)
    got = float((gx.double() * dx).sum() + (gw.double() * dw).sum() + (gb.double() * db).sum())
    ref = R.LossRef(x, w, t, bias, 0.4)
    (_, ex, _, _), (_, ew, _, _), (_, eb) = ref.backward(g)
    bound = float((ex * dx.abs()).sum() + (ew * dw.abs()).sum() + (eb * db.abs()).sum())
    assert abs(got - d1) <= bound + abs(d1 - d2) + 1e-9


def test_the_same_every_time_and_on_another_stream():
    st = torch.cuda.Stream()
    hp = HotPath([1], 4, stream=st.cuda_stream)
    x, w, t, bias, g = _make(13, 400, 6000, 64, BF16, bias=True)
    torch.cuda.synchronize()
    outs = []
    for _ in range(3):
        loss, lse, mean = hp.softmax_loss(x, w, t, bias, 0.1, keep=True)
        outs.append([loss, lse, mean, *hp.softmax_loss_backward(x, w, t, lse, g, mean, bias, 0.1)])
        hp.sync()
    for other in outs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(outs[0], other))


def test_graphs_beside_each_other():
    """Two captured steps of one HotPath, replayed on two streams, with an eager one between them."""
    st = torch.cuda.Stream()
    hp = HotPath([1], 4, stream=st.cuda_stream)
    cases = [_make(20 + i, n, v, d, dt, bias=True) for i, (n, v, d, dt) in enumerate([(300, 5000, 64, F32), (500, 900, 100, F16), (200, 3000, 32, BF16)])]
    torch.cuda.synchronize()

    def step(c):
        x, w, t, bias, g = c
        loss, lse, mean = hp.softmax_loss(x, w, t, bias, 0.2, keep=True)
        out = hp.softmax_loss_backward(x, w, t, lse, g, mean, bias, 0.2)
        return [loss, lse, *out, *hp.softmax_loss_backward(x, w, t, lse, g, None, bias, 0.2)]
    want = [step(c) for c in cases]
    hp.sync()
    graphs, got = [], []
    for c in cases[:2]:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=st):
            got.append(step(c))
    lanes = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        for outs in got:
            for o in outs:
                o.fill_(float("nan"))
        torch.cuda.synchronize()
        for graph, lane in zip(graphs, lanes):
            with torch.cuda.stream(lane):
                graph.replay()
        eager = step(cases[2])
        torch.cuda.synchronize()
        for a, b in zip([*got, eager], want):
            assert all(torch.equal(p, q) for p, q in zip(a, b))


@pytest.mark.parametrize("n,v,d,dtype", [(1500, 9000, 64, F32), (40, 100_000, 32, BF16), (20_000, 200, 128, F16)])
def test_the_largest_call_s_workspace_for_all(hp, n, v, d, dtype):
    x, w, t, bias, g = _make(30, n, v, d, dtype, bias=True)
    whole = B.SoftmaxLoss(n, v, d, t, bias, 0.1, dtype)
    needs = [B.fae_softmax_loss_fwd_workspace_bytes(whole), B.fae_softmax_loss_bwd_workspace_bytes(whole)]
    buf = [torch.full((k + 4096,), 0x5A, dtype=torch.uint8, device="cuda") for k in needs]
    for a, b in ((n, v), (n // 3, v), (n, v // 7), (5, 11), (1, v), (n, 1)):
        xs, ws, ts, bs, gs = x[:a], w[:b], t[:a].clamp(max=b - 1), bias[:b], g[:a]
        what = B.SoftmaxLoss(a, b, d, ts, bs, 0.1, dtype)
        loss, lse, mean = hp.softmax_loss(xs, ws, ts, bs, 0.1, keep=True)
        want = [loss, lse, mean, *hp.softmax_loss_backward(xs, ws, ts, lse, gs, None, bs, 0.1)]
        got = [torch.empty_like(o) for o in want]
        B.fae_softmax_loss_fwd(hp.ctx, what, xs, ws, *got[:3], buf[0][:needs[0]])
        B.fae_softmax_loss_bwd(hp.ctx, what, xs, ws, got[1], None, gs, *got[3:], buf[1][:needs[1]])
        hp.sync()
        assert all(torch.equal(p, q) for p, q in zip(got, want))
    assert all(bool((bf[k:] == 0x5A).all()) for bf, k in zip(buf, needs))


def test_a_table_of_more_than_2_31_values(hp):
    """Rows behind 2^31 values are read and their gradients written where they are."""
    v, d, n = (1 << 31) // 64 + 1000, 64, 3
    w = torch.zeros((v, d), dtype=BF16, device="cuda")
    x = torch.ones((n, d), dtype=BF16, device="cuda")
    at = [v - 1, v - 513, 17]
    for i, r in enumerate(at):
        w[r] = 0.25 + 0.125 * i
    t = torch.tensor(at, dtype=torch.int32, device="cuda")
    loss, lse, mean = hp.softmax_loss(x, w, t, None, 1.0, keep=True)
    gx, gw = hp.softmax_loss_backward(x, w, t, lse, torch.ones(n, device="cuda"), mean, None, 1.0)
    hp.sync()
    z = [64 * (0.25 + 0.125 * i) for i in range(3)]
    total = math.log(sum(math.exp(s) for s in z) + (v - 3))
    assert torch.allclose(lse, torch.full((n,), total, device="cuda"), rtol=1e-5)
    assert torch.allclose(loss, torch.tensor([total - s for s in z], device="cuda"), atol=1e-4)
    p = [math.exp(s - total) for s in z]
    for i, r in enumerate(at):  # three rows with the same probability, one of them has this target
        assert torch.allclose(gw[r].float(), torch.full((d,), 3 * p[i] - 1, device="cuda"), rtol=2 ** -7, atol=1e-6)
        want = sum(p[j] * (0.25 + 0.125 * j) for j in range(3)) - (0.25 + 0.125 * i)
        assert torch.allclose(gx[i].float(), torch.full((d,), want, device="cuda"), rtol=2 ** -6, atol=1e-6)
    rest = math.exp(-total) * 3
    assert torch.allclose(gw[v - 2].float(), torch.full((d,), rest, device="cuda"), rtol=2 ** -7)
    gw[at] = 0
    assert float(gw.float().max()) <= rest * (1 + 2 ** -7) and float(gw.float().min()) >= 0


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,v,d", [(1, 50_021, 64), (64, 33_000, 33), (33, 25_001, 200), (5, 31, 256), (48, 1, 8), (63, 100_000, 16), (65, 9001, 96)])
def test_few_rows_without_mean(hp, n, v, d, dtype):
    """The loss alone: a kernel of its own for up to 64 rows."""
    for with_bias in (False, True):
        x, w, t, bias, _ = _make(n + v + d, n, v, d, dtype, bias=with_bias, pad=with_bias * 3, lead=with_bias)
        if with_bias:
            bias[torch.rand(v, device="cuda") < 0.3] = -math.inf
        ref = R.LossRef(x, w, t, bias, 2.0 / math.sqrt(d))
        loss, lse = hp.softmax_loss(x, w, t, bias, 2.0 / math.sqrt(d))
        hp.sync()
        R.assert_within(lse, ref.lse, ref.dlse, "lse")
        R.assert_within(loss, *ref.loss(), "loss")


@pytest.mark.parametrize("n", [3, 40])
def test_few_rows_and_what_they_may_meet(hp, n):
    x, w, t, bias, _ = _make(7, n, 3000, 40, F32, bias=True)
    t[:] = torch.arange(n, device="cuda") * 7
    t[0] = -1
    bias[:] = torch.linspace(-200, 200, 3000, device="cuda")
    ref = R.LossRef(x, w, t, bias, 0.5)
    loss, lse = hp.softmax_loss(x, w, t, bias, 0.5)
    R.assert_within(lse, ref.lse, ref.dlse, "lse")
    R.assert_within(loss, *ref.loss(), "loss")
    rest = torch.arange(n, device="cuda") != 1
    x[1] = float("nan")
    loss2, lse2 = hp.softmax_loss(x, w, t, bias, 0.5)
    assert torch.equal(loss2[rest], loss[rest]) and math.isnan(float(lse2[1]))
    bias.fill_(-math.inf)
    loss, lse = hp.softmax_loss(x[rest], w, t[rest], bias, 0.5)
    assert bool((lse == -math.inf).all()) and not bool(loss.any())
    hp.sync()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,with_mean", [(20, False), (20, True), (300, False), (300, True), (7000, True)])
def test_classes_that_are_not_offered_may_hold_anything(hp, n, with_mean, dtype):
    """Infinities, NaN and the type's largest value in masked places; a mask of fp32's lowest value is as good as one of infinity."""
    v, d = 3000, 40
    x, w, t, bias, g = _make(n, n, v, d, dtype, bias=True)
    gone = torch.rand(v, device="cuda") < 0.3
    gone[t.clamp(min=0).long()] = False
    clean = w.clone()
    clean[gone] = 0
    bias[gone] = -math.inf

    def calls(w, bias):
        out = hp.softmax_loss(x, w, t, bias, 0.2, keep=with_mean)
        return [*out, *hp.softmax_loss_backward(x, w, t, out[1], g, out[2] if with_mean else None, bias, 0.2)]
    want = calls(clean, bias)
    for fill in (math.nan, math.inf, torch.finfo(dtype).max):
        w[gone] = fill
        assert all(torch.equal(a, b) for a, b in zip(calls(w, bias), want))
    assert all(torch.equal(a, b) for a, b in zip(calls(w, bias.clamp(min=torch.finfo(F32).min)), want))
    hp.sync()


def test_more_rows_than_threads_of_a_grid(hp):
    """2^26 rows and more: kernels with a wave per row walk."""
    n = (1 << 26) + 1000
    x = torch.ones((n, 1), dtype=BF16, device="cuda")
    x[-3:] = 2.0
    w = torch.tensor([[0.5], [1.0], [-1.0]], dtype=BF16, device="cuda")
    t = torch.zeros(n, dtype=torch.int32, device="cuda")
    loss, lse, mean = hp.softmax_loss(x, w, t, keep=True)
    gx, gw = hp.softmax_loss_backward(x, w, t, lse, torch.ones(n, device="cuda"), mean)
    hp.sync()
    for part, value in ((slice(0, n - 3), 1.0), (slice(n - 3, n), 2.0)):
        z = [0.5 * value, value, -value]
        total = math.log(sum(map(math.exp, z)))
        p = [math.exp(s - total) for s in z]
        for got, want, rel in ((lse, total, 1e-5), (loss, total - z[0], 1e-5), (gx, p[0] * 0.5 + p[1] - p[2] - 0.5, 2 ** -6)):
            assert float((got[part].float() - want).abs().max()) <= rel * abs(want)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", [1e-30, 1e-3, 1e4, 1e18])
def test_large_and_small_values(hp, size, dtype):
    """Rows of any size whose scores are of the usual one: x size, w 1 / size."""
    if dtype == F16 and not 1e-4 < size < 1e5:
        pytest.skip("no numbers of fp16")
    for n in (40, 200):
        x, w, t, bias, g = _make(6, n, 100_000 if n == 200 else 500, 48, F32, bias=True)
        x, w = (x * (size if dtype != F16 else 1.0)).to(dtype), (w / size if dtype != F16 else w * size / 100).to(dtype)
        scale = 0.2 if dtype != F16 else 0.2 * 100 / size
        ref = R.LossRef(x, w, t, bias, scale)
        g = g * 1e-3
        _check(hp, x, w, t, bias, g, scale, ref=ref)


def test_values_of_different_sizes(hp):
    """Some rows of the table 2^14 times the others, some columns 2^-12: what is far below the largest keeps its digits."""
    x, w, t, bias, g = _make(9, 256, 70_000, 64, F32)
    w[::7] *= 2.0 ** -14
    w[:, 5] *= 2.0 ** -12
    x[:, 9] *= 2.0 ** -10
    _check(hp, x, w, t, None, g, 0.1)

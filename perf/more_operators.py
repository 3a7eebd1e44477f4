"""What a training step does behind the dense layers, as cases that can be timed and compared: softmax cross entropy over
all rows of a table (next-item prediction: the classes are the table's rows), its gradients, the norm of all
gradients together and clipping by it.

A case is a dict of plain values:
  op       loss (loss and log-sum-exp of every row), grad (the same and the gradients: a training step), norm
           (of all gradients), clip (norm, and gradients scaled to at most max_norm)
  loss and grad:
    rows     rows that are classified (samples)
    classes  rows of the table
    width    values in either
    type     f32, bf16, f16: of rows, table and their gradients
    scale    what the products are multiplied by (one over the temperature)
    bias     whether classes have a bias (the correction for their popularity; some are withdrawn: minus infinity)
    pad      values between the rows of x
  norm and clip:
    tensors  how many gradients
    least, most  values in the smallest and the largest; those between are spread over the logarithm
    type     f32, bf16, f16, or mix: one after the other
    scale    what the gradients are multiplied by first (one over the loss scale)

  z[r, v] = scale * <x[r], w[v]> + bias[v],  lse[r] = log sum_v exp z[r, v],
  loss[r] = lse[r] - z[r, target[r]], 0 where a row has no target (target < 0: a cold row),
  and with g[r] the gradient of loss[r], G[r, v] = g[r] * (exp(z[r, v] - lse[r]) - (v == target[r])):
  gx = scale * G w,  gw = scale * G^T x,  gbias = sum_r G[r].
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
MAX_NORM = 1.0


def _loss(name, op, rows, classes, width, type, scale=1.0, bias=False, pad=0):
    return dict(name=name, op=op, rows=rows, classes=classes, width=width, type=type, scale=scale, bias=bias, pad=pad)


def _list(name, op, tensors, least, most, type, scale=1.0):
    return dict(name=name, op=op, tensors=tensors, least=least, most=most, type=type, scale=scale)


def listed():
    return [
        # serving: how likely one item is for one request, among 200 thousand
        _loss("loss_1x200003x64", "loss", 1, 200_003, 64, "f32", 8.0),
        # a small test batch over a table of a million rows, corrected for popularity
        _loss("loss_48x1000003x32", "loss", 48, 1_000_003, 32, "f32", 10.0, bias=True),
        # evaluation between two swaps: a large batch over a table in the dense layers' type
        _loss("loss_16384x131072x64", "loss", 16384, 131_072, 64, "bf16", 8.0),
        # the smallest training step: the hot samples of a few hundred, a small table
        _loss("grad_300x5003x16", "grad", 300, 5003, 16, "f32", 12.0),
        # behaviour histories: a batch of 2048 over the table of a million rows of 32
        _loss("grad_2048x1000000x32", "grad", 2048, 1_000_000, 32, "f32", 10.0),
        # the dense layers' type, a ragged batch with a gap behind each row, a width that fills no power of two
        _loss("grad_3001x40009x100", "grad", 3001, 40_009, 100, "f16", 6.0, pad=12),
        # a large batch over a table of 100 thousand rows of 64, corrected for popularity
        _loss("grad_16384x100003x64", "grad", 16384, 100_003, 64, "bf16", 8.0, bias=True),
        # the widest rows
        _loss("grad_8192x32768x256", "grad", 8192, 32_768, 256, "bf16", 4.0),
        # gradients of the norms' weights and of a few small layers: latency
        _list("norm_31", "norm", 31, 16, 4096, "f32"),
        # gradients of dense layers and of dozens of tables, 100 million values in more tensors than one launch can name
        _list("norm_300", "norm", 300, 64, 4_000_001, "f32", 1 / 1024),
        # the same for a small model in several types
        _list("clip_40", "clip", 40, 16, 100_003, "mix", 1 / 1024),
        # a large model's, in the dense layers' type, 200 million values
        _list("clip_60", "clip", 60, 64, 38_000_003, "bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges: 1 to 16384 rows over 100 to 2 million classes of width 8 to 256, or 1 to 400 gradients (60 that are clipped)."""
    op = rng.choice(["loss", "grad", "grad", "grad", "norm", "clip"])
    if op in ("norm", "clip"):
        tensors = _log(rng, 1, 400 if op == "norm" else 60)
        least = _log(rng, 1, 4096)
        most = max(least, _log(rng, 4096, 16_000_000))
        type = rng.choice(["f32", "f32", "bf16", "f16", "mix"])
        while sum(_sizes(dict(tensors=tensors, least=least, most=most))) > 200_000_000:
            most = max(least, most * 2 // 3)
        return dict(op=op, tensors=tensors, least=least, most=most, type=type, scale=rng.choice([1.0, 1.0, 1 / 1024, 0.125]))
    type = rng.choice(["f32", "f32", "bf16", "f16"])
    rows, classes, width = _log(rng, 1, 16384), _log(rng, 100, 2_000_000), _log(rng, 8, 256)
    if rng.random() < 0.6:
        width = -(-width // 8) * 8
    while (rows * classes > 2_000_000_000 or rows * classes * width > (60_000_000_000 if type == "f32" else 100_000_000_000) or
           classes * width > 100_000_000):
        if rng.random() < 0.5:
            rows = max(1, rows * 2 // 3)
        else:
            classes = max(100, classes * 2 // 3)
    scale = round(rng.uniform(0.5, 1.2) * 64 / math.sqrt(width), 2)
    return dict(op=op, rows=rows, classes=classes, width=width, type=type, scale=scale, bias=rng.random() < 0.4, pad=rng.choice([0, 0, 8, 13]))


# --------------------------------------------------------------------------------------
def _sizes(case):
    n, lo, hi = case["tensors"], case["least"], case["most"]
    return [int(round(lo * (hi / lo) ** (i / max(n - 1, 1)))) if n > 1 else hi for i in range(n)]


def _types(case):
    names = ["f32", "bf16", "f16"] if case["type"] == "mix" else [case["type"]]
    return [TYPES[names[i % len(names)]] for i in range(case["tensors"])]


def _inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    st = dict(case=case)
    if case["op"] in ("norm", "clip"):
        # values as they are at the end of a backward pass: of another size in every tensor, and times the loss scale
        size = torch.empty(case["tensors"]).uniform_(-4.0, 0.0, generator=torch.Generator().manual_seed(seed)).exp().tolist()
        st["g"] = [torch.empty(n, device="cuda").normal_(0.0, s / case["scale"] / 8, generator=gen).to(t)
                   for n, t, s in zip(_sizes(case), _types(case), size)]
        return st
    n, v, d, t = case["rows"], case["classes"], case["width"], TYPES[case["type"]]
    st["w"] = torch.empty((v, d), device="cuda").uniform_(-0.05, 0.05, generator=gen).to(t)
    target = torch.randint(0, v, (n,), device="cuda", generator=gen)
    # normalised rows, which lean towards their target by what training has reached so far
    lean = torch.empty((n, 1), device="cuda").uniform_(0.0, 12.0, generator=gen) / (case["scale"] * d * 0.05 ** 2 / 3)
    x = torch.empty((n, d), device="cuda").normal_(generator=gen) + lean * st["w"][target].float()
    buf = torch.zeros((n, d + case["pad"]), dtype=t, device="cuda")
    st["x"] = buf[:, :d]
    st["x"].copy_(x)
    st["bias"] = None
    if case["bias"]:
        rank = torch.rand(v, device="cuda", generator=gen)
        st["bias"] = -0.5 * torch.log(rank + 1.0 / v)
        gone = torch.rand(v, device="cuda", generator=gen) < 1 / 64
        gone[target] = False
        st["bias"][gone] = -math.inf
    cold = torch.rand(n, device="cuda", generator=gen) < 1 / 32
    st["target"] = torch.where(cold, -1, target).to(torch.int32)
    weight = 0.5 + torch.rand(n, device="cuda", generator=gen)  # of the samples, in the mean over the batch
    st["g"] = weight * (min(64.0, 1024.0 / n) if case["type"] == "f16" else 1.0 / n)  # fp16: with a loss scale of up to 1024
    return st


_hp = None


def prepare(case, seed):
    st = _inputs(case, seed)
    if not own:
        return st
    from paper_2103_00686_amd import binding as B
    from paper_2103_00686_amd.hotpath import HotPath
    global _hp
    if _hp is None:
        _hp = HotPath([1], 4)  # a program has one, with its tables; these operators take any width
    if case["op"] in ("norm", "clip"):
        norm = torch.empty((), device="cuda")
        if case["op"] == "norm":
            st["calls"] = [_hp.prepare_gradient_norm(st["g"], norm, case["scale"])]
            st["out"] = norm
        else:
            out = [torch.empty_like(g) for g in st["g"]]
            st["calls"] = [_hp.prepare_clip_gradients(st["g"], MAX_NORM, norm, case["scale"], out)]
            st["out"] = [norm, *out]
        return st
    n, v, d = case["rows"], case["classes"], case["width"]
    what = B.SoftmaxLoss(n, v, d, st["target"], st["bias"], case["scale"], TYPES[case["type"]])
    loss, lse = torch.empty((2, n), device="cuda")
    if case["op"] == "loss":
        st["calls"] = [_hp.prepare_softmax_loss(what, st["x"], st["w"], loss, lse)]
        st["out"] = [loss, lse]
        return st
    mean = torch.empty((n, d), device="cuda")
    gx, gw = torch.empty((n, d), dtype=st["x"].dtype, device="cuda"), torch.empty_like(st["w"])
    gbias = torch.empty(v, device="cuda") if case["bias"] else None
    st["calls"] = [_hp.prepare_softmax_loss(what, st["x"], st["w"], loss, lse, mean),
                   _hp.prepare_softmax_loss_backward(what, st["x"], st["w"], lse, st["g"], gx, gw, gbias, mean)]
    st["out"] = [loss, lse, gx, gw] + ([gbias] if case["bias"] else [])
    return st


def run(st):
    if own:
        for call in st["calls"]:
            call()
        return st["out"]
    return _plain(st)


# -- the plain form: elementary torch operations in 32 bits, long sums in 64 -------------------
def _plain(st):
    case = st["case"]
    if case["op"] in ("norm", "clip"):
        squares = torch.stack([torch.square(g.float()).sum(dtype=torch.float64) for g in st["g"]])
        norm = (squares.sum().sqrt() * case["scale"]).float()
        if case["op"] == "norm":
            return norm
        factor = torch.where(norm > MAX_NORM, MAX_NORM / norm, torch.ones_like(norm)) * case["scale"]
        return [norm] + [(g.float() * factor).to(g.dtype) for g in st["g"]]
    n = case["rows"]
    x, w, t = st["x"].float(), st["w"].float(), st["target"].long()
    z = x @ w.t()
    z *= case["scale"]
    if case["bias"]:
        z += st["bias"]
    most = z.max(1, keepdim=True).values
    at = torch.arange(n, device="cuda"), t.clamp(min=0)
    zt = z[at]
    z -= most
    z.exp_()
    s = z.sum(1, keepdim=True)
    lse = (most + s.log())[:, 0]
    loss = torch.where(t >= 0, lse - zt, 0.0)
    if case["op"] == "loss":
        return [loss, lse]
    z /= s
    z[at] -= 1.0
    z *= torch.where(t >= 0, st["g"], 0.0)[:, None]
    some = 1 << 14  # classes whose products are summed in 32 bits; a million of them would lose three digits
    gx = torch.stack([zc @ wc for zc, wc in zip(z.split(some, 1), w.split(some))]).sum(0, dtype=torch.float64).float()
    gw = z.t() @ x
    dtype = st["x"].dtype
    out = [loss, lse, gx.mul_(case["scale"]).to(dtype), gw.mul_(case["scale"]).to(dtype)]
    return out + [z.sum(0)] if case["bias"] else out


# -- the definition in 64 bits, some classes at a time ---------------------------------------
def exact(case, seed):
    st = _inputs(case, seed)
    if case["op"] in ("norm", "clip"):
        norm = torch.stack([torch.linalg.vector_norm(g.double()) for g in st["g"]])
        norm = (norm * norm).sum().sqrt() * case["scale"]
        if case["op"] == "norm":
            return norm
        factor = case["scale"] * min(1.0, MAX_NORM / float(norm))
        return [norm] + [g.double() * factor for g in st["g"]]
    n, v, d = case["rows"], case["classes"], case["width"]
    x, t = st["x"].double() * case["scale"], st["target"].long()
    some = max(1024, (1 << 27) // n)

    def logits():
        for v0 in range(0, v, some):
            v1 = min(v, v0 + some)
            w = st["w"][v0:v1].double()
            z = torch.mm(x, w.t().contiguous())
            yield v0, v1, w, (z + st["bias"][v0:v1].double() if case["bias"] else z)
    parts = [torch.logsumexp(z, 1) for _, _, _, z in logits()]
    lse = torch.logsumexp(torch.stack(parts), 0)
    known = t >= 0
    zt = (x * st["w"][t.clamp(min=0)].double()).sum(1)
    if case["bias"]:
        zt = zt + st["bias"][t.clamp(min=0)].double()
    loss = (lse - zt) * known
    if case["op"] == "loss":
        return [loss, lse]
    g = st["g"].double() * known
    gx = torch.zeros((n, d), dtype=torch.float64, device="cuda")
    gw = torch.empty((v, d), dtype=torch.float64, device="cuda")
    gbias = torch.empty(v, dtype=torch.float64, device="cuda")
    for v0, v1, w, z in logits():
        p = torch.exp(z - lse[:, None])
        rows = torch.nonzero(known & (t >= v0) & (t < v1))[:, 0]
        p[rows, t[rows] - v0] -= 1.0
        p *= g[:, None]
        gx += p @ w
        gw[v0:v1] = torch.mm(p.t().contiguous(), x)
        gbias[v0:v1] = p.sum(0)
    out = [loss, lse, gx * case["scale"], gw]
    return out + [gbias] if case["bias"] else out


def work(case):
    """Of a training step: the products are computed once, and once each for the two gradients."""
    if case["op"] in ("norm", "clip"):
        values = sum(_sizes(case))
        size = sum(n * t.itemsize for n, t in zip(_sizes(case), _types(case)))
        return {"bytes": size + 4, "flops": 2 * values} if case["op"] == "norm" else {"bytes": 2 * size + 4, "flops": 3 * values}
    n, v, d, size = case["rows"], case["classes"], case["width"], TYPES[case["type"]].itemsize
    bias = 4 * v if case["bias"] else 0
    if case["op"] == "loss":
        return {"bytes": (n + v) * d * size + bias + 12 * n, "flops": n * v * (2 * d + 4)}
    return {"bytes": 2 * (n + v) * d * size + 2 * bias + 16 * n, "flops": n * v * (6 * d + 8)}

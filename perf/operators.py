"""Row normalisation and dropout between the pooled forward and the dense layers, as cases that can
be timed and compared: layer norm and its backward (per table's pooled row, or over a whole sample),
dropout and its backward, and the two together in one pass each way.

A case is a dict of plain values:
  op       norm, norm_grad, drop, drop_grad
  rows     samples
  parts    rows of a sample that are normalised on their own (tables); 1 = the whole sample
  width    values in such a row
  x, y     types: f32, bf16, f16 (x: what is normalised, y: what the dense layers read; of a
           gradient gy has y's type and gx has x's)
  p        share that dropout drops (0 for a norm without dropout)
  affine   norm: whether it has weights
  pad      values between the samples of x (drop_grad: of gy), as in a row stride above parts * width
  counter  whether the generator's offset is read from device memory (captured steps)

The mask of dropout: Philox4x32-10 with the counter (c >> 3, r, offset) and the seed as its key gives
eight 16-bit pieces for eight columns c of row r, low halves first; a value goes where its piece is
below T = round(65536 p), and what stays is multiplied by 65536 / (65536 - T).
"""
import math

import torch

own = False

EPS = 1e-5
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _case(name, op, rows, parts, width, x, y, p=0.0, affine=True, pad=0, counter=False):
    return dict(name=name, op=op, rows=rows, parts=parts, width=width, x=x, y=y, p=p, affine=affine, pad=pad, counter=counter)


def listed():
    return [
        # serving one request: the pooled rows of 26 tables
        _case("norm_1x26x64", "norm", 1, 26, 64, "f32", "f32"),
        # every table's pooled row of the Terabyte-like batch, bench.py's headline workload
        _case("norm_16384x26x64", "norm", 16384, 26, 64, "f32", "f32"),
        # a large ragged batch of the same tables, with dropout and in the dense layers' type
        _case("norm_drop_50001x26x64", "norm", 50001, 26, 64, "f32", "bf16", p=0.1),
        # the smallest training step: the hot samples of a thousand, one table
        _case("norm_grad_717x16", "norm_grad", 717, 1, 16, "f32", "f32"),
        # behaviour histories: a width that fills no power of two, pooled rows with a gap behind each sample
        _case("norm_grad_6007x4x100", "norm_grad", 6007, 4, 100, "f32", "f32", pad=20),
        # the headline batch's backward
        _case("norm_grad_16384x26x64", "norm_grad", 16384, 26, 64, "f32", "f32"),
        # the large ragged batch's backward: fp32 rows, gradients from layers in bfloat16, dropout
        _case("norm_drop_grad_50001x26x64", "norm_grad", 50001, 26, 64, "f32", "bf16", p=0.1),
        # whole samples of 26 tables of 64 as one row each, in the dense layers' type
        _case("norm_grad_4096x1664", "norm_grad", 4096, 1, 1664, "bf16", "bf16"),
        # wide rows, as after a dense layer
        _case("norm_grad_16384x8192", "norm_grad", 16384, 1, 8192, "bf16", "bf16"),
        # a small batch of three tables of 32: latency
        _case("drop_2048x96", "drop", 2048, 1, 96, "f32", "f32", p=0.5),
        # the large ragged batch into the dense layers' type
        _case("drop_50001x1664", "drop", 50001, 1, 1664, "f32", "bf16", p=0.1),
        # gradients of eight tables of 128, in a captured step: the offset is in device memory
        _case("drop_grad_65536x1024", "drop_grad", 65536, 1, 1024, "f16", "f16", p=0.2, counter=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges: up to 64 tables of up to 256 values, or one row of up to 16384."""
    op = rng.choice(["norm", "norm_grad", "norm_grad", "drop", "drop_grad"])
    x, y = rng.choice([("f32", "f32"), ("f32", "f32"), ("f32", "bf16"), ("f32", "f16"), ("bf16", "bf16"), ("f16", "f16")])
    parts = rng.choice([1, 1, 2, 3, 5, 8, 13, 26, 40, 64]) if op.startswith("norm") else 1
    width = _log(rng, 8, 256) if parts > 1 else _log(rng, 8, 16384)
    if rng.random() < 0.6:
        width = -(-width // 8) * 8
    rows = _log(rng, 1, 131072)
    while rows * parts * width > 80_000_000:
        rows = max(1, rows * 2 // 3)
    p = rng.choice([0.1, 0.2, 0.5]) if op.startswith("drop") else rng.choice([0.0, 0.0, 0.1, 0.25])
    affine = op.startswith("norm") and rng.random() < 0.85
    pad = rng.choice([0, 0, 0, 8, 13])
    return dict(op=op, rows=rows, parts=parts, width=width, x=x, y=y, p=p, affine=affine, pad=pad, counter=p > 0 and rng.random() < 0.3)


# --------------------------------------------------------------------------------------
def _inputs(case, seed):
    """Pooled rows (sums of a few embeddings of +-0.05, some bags empty), gradients, weights, seeds."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    n, parts, w = case["rows"], case["parts"], case["width"]
    tx, ty = TYPES[case["x"]], TYPES[case["y"]]
    st = dict(case=case, x=None, gy=None, gamma=None, beta=None)

    def tensor(dtype, values, pad=0):
        buf = torch.zeros((n, parts * w + pad), dtype=dtype, device="cuda")
        view = buf[:, :parts * w].unflatten(1, (parts, w))
        view.copy_(values)
        return view

    if case["op"] != "drop_grad":
        v = torch.empty((n, parts, w), device="cuda").uniform_(-0.1, 0.1, generator=gen)
        bags = torch.rand((n, parts, 1), device="cuda", generator=gen)
        st["x"] = tensor(tx, v.mul_((bags > 1 / 64).float() * (0.5 + bags)), case["pad"])
        del v
    if case["op"].endswith("_grad"):
        st["gy"] = tensor(ty, torch.empty((n, parts, w), device="cuda").normal_(generator=gen), case["pad"] if st["x"] is None else 0)
    if case["affine"]:
        st["gamma"] = torch.empty((parts, w), device="cuda").normal_(1.0, 0.2, generator=gen)
        st["beta"] = torch.empty((parts, w), device="cuda").normal_(0.0, 0.2, generator=gen)
    st["seed"] = (seed * 0x9E3779B97F4A7C15 + 12345) % (1 << 64)
    st["offset"] = (1 << 32) - 3 + seed % 7
    st["counter"] = torch.full((1,), 5 + seed % 3, dtype=torch.int64, device="cuda") if case["counter"] else None
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
    op, n, parts, w = case["op"], case["rows"], case["parts"], case["width"]
    tx, ty = TYPES[case["x"]], TYPES[case["y"]]
    drop = B.Drop(case["p"], st["seed"], st["offset"], st["counter"]) if case["p"] > 0 else None
    fwd = not op.endswith("_grad")
    out = torch.empty((n, parts, w), dtype=ty if fwd else tx, device="cuda")
    if op == "drop":
        st["call"], st["out"] = _hp.prepare_dropout(drop, st["x"], out), out
    elif op == "drop_grad":
        st["call"], st["out"] = _hp.prepare_dropout_backward(drop, st["gy"], out), out
    else:
        norm = B.Norm(n, parts, w, st["gamma"], st["beta"], EPS, tx, ty)
        if fwd:
            st["call"], st["out"] = _hp.prepare_layer_norm(norm, st["x"], out, drop), out
        else:
            dg, db = (torch.empty((parts, w), device="cuda") if case["affine"] else None for _ in range(2))
            st["call"] = _hp.prepare_layer_norm_backward(norm, st["x"], st["gy"], out, dg, db, drop)
            st["out"] = [out, dg, db] if case["affine"] else out
    return st


def run(st):
    if own:
        st["call"]()
        return st["out"]
    return _plain(st)


# -- the plain form: elementary torch operations in 32 bits ----------------------------------
def _keep(st):
    """The values that dropout keeps, [rows * parts, width], and what they are multiplied by."""
    case = st["case"]
    n, w, m = case["rows"] * case["parts"], case["width"], 0xFFFFFFFF
    off = st["offset"] + (st["counter"] if st["counter"] is not None else 0)
    groups = (w + 7) // 8
    c0 = torch.arange(groups, device="cuda").expand(n, groups)
    c1 = torch.arange(n, device="cuda")[:, None].expand(n, groups)
    c2 = (torch.zeros_like(c0) + off) & m
    c3 = ((torch.zeros_like(c0) + off) >> 32) & m
    k0, k1 = st["seed"] & m, st["seed"] >> 32
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57  # 64-bit products; the sign bit goes with the mask
        c0, c1, c2, c3 = ((b >> 32) & m) ^ c1 ^ k0, b & m, ((a >> 32) & m) ^ c3 ^ k1, a & m
        k0, k1 = (k0 + 0x9E3779B9) & m, (k1 + 0xBB67AE85) & m
    words = torch.stack([c0, c1, c2, c3], 2)
    pieces = torch.stack([words & 0xFFFF, words >> 16], 3).reshape(n, groups * 8)[:, :w]
    t = int(round(case["p"] * 65536))
    return (pieces >= t).reshape(case["rows"], case["parts"], w), 65536.0 / (65536 - t)


def _dropped(st, v):
    keep, scale = _keep(st)
    return torch.where(keep, v * scale, 0.0)


def _plain(st):
    case = st["case"]
    tx, ty = TYPES[case["x"]], TYPES[case["y"]]
    if case["op"] == "drop":
        return _dropped(st, st["x"].float()).to(ty)
    if case["op"] == "drop_grad":
        return _dropped(st, st["gy"].float()).to(tx)
    x = st["x"].float()
    d = x - x.mean(2, keepdim=True)
    s = 1.0 / torch.sqrt((d * d).mean(2, keepdim=True) + EPS)
    h = d * s
    if case["op"] == "norm":
        v = h * st["gamma"] + st["beta"] if case["affine"] else h
        return (_dropped(st, v) if case["p"] > 0 else v).to(ty)
    g = st["gy"].float()
    if case["p"] > 0:
        g = _dropped(st, g)
    a = g * st["gamma"] if case["affine"] else g
    gx = (s * (a - a.mean(2, keepdim=True) - h * (a * h).mean(2, keepdim=True))).to(tx)
    if not case["affine"]:
        return gx
    return [gx, (g * h).sum(0, dtype=torch.float64).float(), g.sum(0, dtype=torch.float64).float()]


# -- the definition in 64 bits -------------------------------------------------------------
def _mulhilo(a, b):
    """High and low word of 32-bit products, by 16-bit parts."""
    ah, al, bh, bl = a >> 16, a & 0xFFFF, b >> 16, b & 0xFFFF
    mid = al * bh + ((al * bl) >> 16)
    low = ah * bl + (mid & 0xFFFF)
    return ah * bh + (mid >> 16) + (low >> 16), (a * b) & 0xFFFFFFFF


def _factors(case, st):
    """What each value is multiplied by: 0 where it is dropped."""
    n, w = case["rows"] * case["parts"], case["width"]
    off = st["offset"] + (int(st["counter"]) if st["counter"] is not None else 0)
    t = int(round(case["p"] * 65536))
    out = torch.empty((n, w), dtype=torch.float64, device="cuda")
    col = torch.arange(0, w, 8, device="cuda")
    step = max(1, (1 << 23) // max(1, col.numel()))
    for r0 in range(0, n, step):
        r = torch.arange(r0, min(n, r0 + step), device="cuda")
        ctr = [(col // 8).repeat(len(r)), r.repeat_interleave(len(col)), torch.tensor(off & 0xFFFFFFFF, device="cuda"),
               torch.tensor(off >> 32, device="cuda")]
        key = [st["seed"] & 0xFFFFFFFF, st["seed"] >> 32]
        for rnd in range(10):
            h0, l0 = _mulhilo(ctr[0], 0xD2511F53)
            h1, l1 = _mulhilo(ctr[2], 0xCD9E8D57)
            ctr = [h1 ^ ctr[1] ^ ((key[0] + rnd * 0x9E3779B9) & 0xFFFFFFFF), l1,
                   h0 ^ ctr[3] ^ ((key[1] + rnd * 0xBB67AE85) & 0xFFFFFFFF), l0]
        for j in range(min(8, w)):
            piece = (ctr[j // 2] >> (16 * (j % 2))) & 0xFFFF
            f = torch.where(piece < t, 0.0, 65536.0 / (65536 - t)).to(torch.float64)
            cols = col[col + j < w] + j
            out[r0:r0 + len(r)][:, cols] = f.reshape(len(r), len(col))[:, :len(cols)]
    return out.reshape(case["rows"], case["parts"], w)


def exact(case, seed):
    st = _inputs(case, seed)
    f = _factors(case, st) if case["p"] > 0 else None
    if case["op"] == "drop":
        return st["x"].double() * f
    if case["op"] == "drop_grad":
        return st["gy"].double() * f
    x = st["x"].double()
    w = case["width"]
    mu = x.sum(2, keepdim=True) / w
    var = ((x - mu) ** 2).sum(2, keepdim=True) / w
    h = (x - mu) / (var + EPS).sqrt()
    gamma = st["gamma"].double() if case["affine"] else torch.ones((), dtype=torch.float64, device="cuda")
    if case["op"] == "norm":
        y = h * gamma
        if case["affine"]:
            y += st["beta"].double()
        return y if f is None else y * f
    g = st["gy"].double()
    if f is not None:
        g = g * f
    a = g * gamma
    gx = (a - (a.sum(2, keepdim=True) + h * (a * h).sum(2, keepdim=True)) / w) / (var + EPS).sqrt()
    return [gx, (g * h).sum(0), g.sum(0)] if case["affine"] else gx


def work(case):
    n = case["rows"] * case["parts"] * case["width"]
    bx, by = TYPES[case["x"]].itemsize, TYPES[case["y"]].itemsize
    weights = 4 * case["parts"] * case["width"] if case["affine"] else 0
    rnd = 14 if case["p"] > 0 else 0  # ten rounds of ten operations for eight values, a comparison, a product
    if case["op"].startswith("drop"):
        return {"bytes": n * (bx + by), "flops": n * rnd}
    if case["op"] == "norm":
        return {"bytes": n * (bx + by) + 2 * weights, "flops": n * (8 + rnd)}
    return {"bytes": n * (2 * bx + by) + 3 * weights, "flops": n * (17 + rnd)}

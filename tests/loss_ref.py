"""Softmax cross entropy over a table's rows from its definition in 64 bits, with a bound for what the kernels' arithmetic may add.

Bounds (u = 2^-24; h = half a step of the type, finfo.eps / 2; N = 1 product per pair of 16-bit values, 6 per pair of fp32 values, which are
three bf16 numbers each).  A matrix instruction adds 16 products to a sum with at most 16 roundings, so a product of `width` values
errs by at most u (N width + 8) A with A = sum |x w| (the 8: what the six products leave out, 2^-23 A, and the factor), a score by
  dz = u (|scale| (N width + 8) A + 4 |z| + 2 |bias|),
lse by the probabilities' mean of dz, by its sum over the classes (two additions per 32 classes and lane, 64 to join lanes and parts), by
two units of 2^z and by the rounding of z - reference, which is below |z - lse| + 1:
  dlse = sum p dz + u (V / 16 + 64 + sum p (8 + 2 |z - lse|) + 4 |lse|).
A probability's relative error is e = dz + dlse + u (8 + 2 |z - lse|) (as a factor, exp(e) - 1).  Entering a product it is
rounded to the type, by h of itself (fp32: by 2^-24, as three bf16 numbers); sums of M such terms take at most N M + 64 roundings of the
sum of their absolute values.  A 16-bit result is off by half a step more.  fp16 probabilities have a smallest step: they
are multiplied by 2^12 at least 1 / 2 of the largest, so each is off by 2^-36 of that at most.  Of the other types, 2^z and the parts of a
probability below fp32's smallest normal number, 2^-126, are lost: each is off by 2^-125 at most.

Beside this worst case, fp32 results are held to what independent roundings add up to: one of at most 2 units per
matrix instruction, so 2 sqrt(number of instructions) + 16 units of the terms' absolute sum, in root mean square.  The terms here are
|g| (p + (v == target)): p is rounded before the 1 is taken off (one class: p = 1 + 2^-23 leaves 2^-23 where p - 1 is 0).
"""
import numpy as np
import torch

U = 2.0 ** -24
F = torch.float64


def half_step(ref, dtype):
    f = torch.finfo(dtype)
    return torch.nan_to_num(ref, posinf=0, neginf=0).abs() * (f.eps / 2) + f.smallest_normal * f.eps / 2


class LossRef:
    def __init__(self, x, w, targets, bias=None, scale=1.0):
        self.dtype = x.dtype
        self.N = 6 if x.dtype == torch.float32 else 1
        self.h = U if x.dtype == torch.float32 else torch.finfo(x.dtype).eps / 2
        self.tiny = 2.0 ** -36 if x.dtype == torch.float16 else 2.0 ** -125
        self.x, self.w = x.double(), w.double()
        self.scale = float(np.float32(scale))
        self.n, self.v, self.d = x.shape[0], w.shape[0], x.shape[1]
        t = targets.long()
        self.known = (t >= 0) & (t < self.v)
        self.t = t.clamp(0, self.v - 1)
        z = self.scale * (self.x @ self.w.t().contiguous())
        A = self.x.abs() @ self.w.abs().t().contiguous()
        b = torch.zeros(self.v, dtype=F, device=x.device) if bias is None else bias.double()
        self.bias = bias
        self.z = z + b
        fine = torch.isfinite(self.z)
        self.dz = torch.where(fine, U * (abs(self.scale) * (self.N * self.d + 8) * A + 4 * z.abs() + 2 * torch.nan_to_num(b, neginf=0).abs()), torch.zeros((), dtype=F, device=x.device))
        self.empty = ~fine.any(1) if self.n else self.known
        self.lse = torch.logsumexp(self.z, 1)
        off = torch.where(fine, self.z - self.lse[:, None], torch.full((), -float("inf"), dtype=F, device=x.device))
        self.p = torch.exp(off)
        far = torch.nan_to_num(off, neginf=0).abs()
        self.dlse = (self.p * self.dz).sum(1) + U * (self.v / 16 + 64 + (self.p * (8 + 2 * far)).sum(1) + 4 * torch.nan_to_num(self.lse, neginf=0).abs())
        self.e = torch.expm1(self.dz + self.dlse[:, None] + U * (8 + 2 * far))
        self.hot = torch.zeros_like(self.z)
        if self.n:
            self.hot[torch.arange(self.n, device=x.device), self.t] = 1.0
        self.live = self.known & ~self.empty

    def loss(self):
        zt = (self.z * 1.0).gather(1, self.t[:, None])[:, 0] if self.n else self.lse
        dt = self.dz.gather(1, self.t[:, None])[:, 0] if self.n else self.dlse
        zero = torch.zeros_like(self.lse)
        return (torch.where(self.live, self.lse - zt, zero),
                torch.where(self.live, self.dlse + dt + 4 * U * (self.lse.abs() + torch.nan_to_num(zt, neginf=0).abs()), zero))

    def mean(self):
        others = self.p * (1 - self.hot * self.known[:, None])
        ref = others @ self.w
        err = (others * (self.e + self.h)) @ self.w.abs() + U * (self.N * self.v + 64) * (others @ self.w.abs()) + self.tiny * self.w.abs().sum(0)
        return ref, err

    def backward(self, gloss, out_dtype=None):
        """((gx, its bound, terms, instructions), the same of gw, (gbias, its bound))"""
        out_dtype = out_dtype or self.dtype
        g = torch.where(self.live, gloss.double(), torch.zeros((), dtype=F, device=gloss.device))[:, None]
        q = torch.where(self.live[:, None], self.p - self.hot, torch.zeros((), dtype=F, device=gloss.device))
        x = torch.where(self.live[:, None], self.x, torch.zeros((), dtype=F, device=gloss.device))
        e = torch.nan_to_num(self.e, posinf=0)
        p = torch.where(self.live[:, None], self.p, torch.zeros((), dtype=F, device=gloss.device))
        G, s = g * q, abs(self.scale)
        dq = p * e + U * self.hot * 8 + q.abs() * (self.h + 4 * U)  # of p - (v == target), as it enters a product
        gx = self.scale * (G @ self.w)
        tx = s * (G.abs() @ self.w.abs())
        dx = s * ((g.abs() * dq) @ self.w.abs()) + U * (self.N * self.v + 80) * tx + s * g.abs() * self.tiny * self.w.abs().sum(0)
        gw = self.scale * (G.t().contiguous() @ x)
        tw = s * (G.abs().t().contiguous() @ x.abs())
        both = g.abs() * (p + self.hot)
        rx, rw = s * (both @ self.w.abs()), s * (both.t().contiguous() @ x.abs())
        most = g.abs().max() if self.n else 0.0
        dw = s * ((g.abs() * dq).t().contiguous() @ x.abs()) + U * (self.N * self.n + 80) * tw + s * most * self.tiny * x.abs().sum(0)
        gb = G.sum(0)
        db = (g.abs() * dq).sum(0) + U * (self.n + 80) * G.abs().sum(0) + most * self.tiny * self.n
        if out_dtype != torch.float32:
            dx, dw = dx + half_step(gx.abs() + dx, out_dtype), dw + half_step(gw.abs() + dw, out_dtype)
        return (gx, dx, rx, self.N * self.v / 16 + self.N * self.d / 16), (gw, dw, rw, self.N * self.n / 16 + self.N * self.d / 16), (gb, db)


def assert_within(got, ref, err, what):
    got = got.double()
    fine = torch.isfinite(ref)
    assert torch.equal(torch.isnan(got), torch.isnan(ref)), what
    assert torch.equal(got[~fine & ~torch.isnan(ref)], ref[~fine & ~torch.isnan(ref)]), what
    far = torch.where(fine, (got - ref).abs() - err - 1e-40, torch.full((), -1.0, dtype=F, device=got.device))
    assert bool((far <= 0).all()), f"{what}: {int((far > 0).sum())} of {far.numel()} too far, worst {float(far.max()):.3e} at {int(far.argmax())}"


def assert_rms(got, ref, terms, instructions, what):
    err = (got.double() - ref).square().mean().sqrt()
    most = U * (2 * instructions ** 0.5 + 16) * terms.square().mean().sqrt()
    assert float(err) <= float(most) + 1e-40, f"{what}: rms {float(err):.3e}, at most {float(most):.3e}"

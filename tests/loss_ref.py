"""Softmax cross entropy over a table's rows from its definition in 64 bits, with a bound for what the kernels' arithmetic may add.

Bounds (u = 2^-24; h = half a step of the type, finfo.eps / 2; N products per pair of values: 1 of 16 bits, up to 6 of fp32, whose values
are three bf16 numbers or, after a power of two that brings the largest of all to 2^14 .. 2^15, two fp16 numbers).  Of fp32's
products at most 2^-22 for each operand and 2^-22 for what is not multiplied is left out, 12 u, and of values 2^-18 below
the largest half a step of fp16, 2^-25 where the largest is 2^14: m = 2^-38 of it.  A matrix instruction adds 16 products
to a sum with at most 16 roundings, so a product of `width` values errs by at most u (N width + 16) A + m's with A = sum |x w|, a score by
  dz = u (|scale| (N width + 16) A + 4 |z| + 2 |bias|) + |scale| (m_w sum |x| + m_x sum |w|),
lse by the probabilities' mean of dz, by its sum over the classes (two additions per 32 classes and lane, 64 to join lanes and parts), by
two units of 2^z and by the rounding of z - reference, which is below |z - lse| + 1:
  dlse = sum p dz + u (V / 16 + 64 + sum p (8 + 2 |z - lse|) + 4 |lse|).
A probability's relative error is e = dz + dlse + u (8 + 2 |z - lse|) (as a factor, exp(e) - 1).  Entering a product it is
rounded to the type, by h of itself (fp32: 16 u as above); sums of M such terms take at most N M + 64 roundings of the
sum of their absolute values.  A 16-bit result is off by half a step more.  fp16 probabilities have a smallest step: the
largest is at least 2^9 (with the gradients 2^14), and half a step is 2^-25: each is off by 2^-34 of the largest at most.  Of bf16 numbers, 2^z and the parts of a
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
        self.h = 16 * U if x.dtype == torch.float32 else torch.finfo(x.dtype).eps / 2
        self.tiny = 2.0 ** -125 if x.dtype == torch.bfloat16 else 2.0 ** -34
        self.x, self.w = x.double(), w.double()
        self.scale = float(np.float32(scale))
        self.n, self.v, self.d = x.shape[0], w.shape[0], x.shape[1]
        t = targets.long()
        self.known = (t >= 0) & (t < self.v)
        self.t = t.clamp(0, self.v - 1)
        z = self.scale * (self.x @ self.w.t().contiguous())
        A = self.x.abs() @ self.w.abs().t().contiguous()
        b = torch.zeros(self.v, dtype=F, device=x.device) if bias is None else bias.double()
        wide = x.dtype == torch.float32
        self.mx = 2.0 ** -38 * float(torch.nan_to_num(self.x, posinf=0, neginf=0).abs().max()) if wide and self.n else 0.0
        self.mw = 2.0 ** -38 * float(torch.nan_to_num(self.w, posinf=0, neginf=0).abs().max()) if wide else 0.0
        off = self.mw * self.x.abs().sum(1)[:, None] + self.mx * self.w.abs().sum(1)
        self.bias = bias
        self.z = z + b
        fine = torch.isfinite(self.z)
        self.dz = torch.where(fine, U * (abs(self.scale) * (self.N * self.d + 16) * A + 4 * z.abs() + 2 * torch.nan_to_num(b, neginf=0).abs()) + abs(self.scale) * off, torch.zeros((), dtype=F, device=x.device))
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
        wt = self.w[self.t] * self.known[:, None]
        ref = others @ self.w - others.sum(1)[:, None] * wt
        both = others @ self.w.abs() + others.sum(1)[:, None] * wt.abs()
        err = (others * (self.e + self.h)) @ self.w.abs() + (others * self.e).sum(1)[:, None] * wt.abs()
        return ref, err + U * (self.N * self.v + 64) * both + self.tiny * (self.w.abs().sum(0) + self.v * wt.abs()) + self.mw

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
        dx = s * ((g.abs() * dq) @ self.w.abs()) + U * (self.N * self.v + 80) * tx + s * g.abs() * (self.tiny * self.w.abs().sum(0) + 2 * self.mw)
        gw = self.scale * (G.t().contiguous() @ x)
        tw = s * (G.abs().t().contiguous() @ x.abs())
        both = g.abs() * (p + self.hot)
        rx, rw = s * (both @ self.w.abs()), s * (both.t().contiguous() @ x.abs())
        most = g.abs().max() if self.n else 0.0
        dw = s * ((g.abs() * dq).t().contiguous() @ x.abs()) + U * (self.N * self.n + 80) * tw + s * (most * self.tiny * x.abs().sum(0) + self.mx * G.abs().sum(0)[:, None])
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

"""Layer norm and dropout from their definitions in 64 bits, with a bound for what fp32 arithmetic may add.

Bounds (u = 2^-24, one rounding of fp32; W the row's width).  A row's sums run through chains of at most
k = ceil(W / 64) + 16 additions (a row is shared by 64 lanes and more, or by W / 4 where it is shorter, then joined in
pairs), so a sum of terms t errs by at most k u sum|t|.  With m any first mean and d = x - m, the mean of d has the error
(k + 2) u mean|d| <= (k + 2) u sigma, so a centred value errs by u |d| + u |c| + (k + 2) u sigma; the variance by
(k + 4) u of itself, its root's reciprocal by half of that and three roundings.  For h = (x - mean) / sigma:
  dh <= u ((k / 2 + 8) |h| + k + 4)
and a result of a few products and additions more adds a rounding of each term.  A result of a 16-bit type
is off by half a step more, eps / 2 of its value (and half of the smallest step below the normal range).
"""
import numpy as np
import torch

U = 2.0 ** -24


def philox_numbers(rows, width, seed, offset):
    """uint16 [rows, width]: the numbers that decide, by 64-bit integer arithmetic on the host."""
    groups = (width + 7) // 8
    m = np.uint64(0xFFFFFFFF)
    sh = np.uint64(32)
    c0, c1 = (a.astype(np.uint64).ravel() for a in np.meshgrid(np.arange(groups), np.arange(rows)))
    c2 = np.full_like(c0, offset & 0xFFFFFFFF)
    c3 = np.full_like(c0, (offset >> 32) & 0xFFFFFFFF)
    k0, k1 = seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF
    for _ in range(10):
        a, b = c0 * np.uint64(0xD2511F53), c2 * np.uint64(0xCD9E8D57)
        c0, c1, c2, c3 = (b >> sh) ^ c1 ^ np.uint64(k0), b & m, (a >> sh) ^ c3 ^ np.uint64(k1), a & m
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    words = np.stack([c0, c1, c2, c3], 1).astype(np.uint32)
    return words.view(np.uint16).reshape(rows, groups * 8)[:, :width]


def keep_and_scale(rows, width, p, seed, offset=0):
    """bool [rows, width] of kept values, and the factor of these."""
    t = int(round(p * 65536))
    keep = philox_numbers(rows, width, seed, offset).astype(np.int64) >= t
    return torch.from_numpy(keep), (65536.0 / (65536 - t) if t < 65536 else 0.0)


def half_step(ref, dtype):
    f = torch.finfo(dtype)
    return ref.abs() * (f.eps / 2) + f.smallest_normal * f.eps / 2


class NormRef:
    """x, gy: [n, parts, width] in their types; gamma, beta: [parts, width] fp32 or None; keep, scale: dropout's."""

    def __init__(self, x, gamma, beta, eps, keep=None, scale=1.0):
        self.x, self.w = x.double(), x.shape[-1]
        self.k = -(-self.w // 64) + 16
        self.gamma = torch.ones_like(self.x[0]) if gamma is None else gamma.double().reshape(x.shape[1:])
        self.beta = torch.zeros_like(self.x[0]) if beta is None else beta.double().reshape(x.shape[1:])
        self.keep, self.scale = keep, scale
        eps = float(np.float32(eps))
        mu = self.x.mean(-1, keepdim=True)
        self.s = 1.0 / (((self.x - mu) ** 2).mean(-1, keepdim=True) + eps).sqrt()
        self.h = (self.x - mu) * self.s
        self.dh = U * ((self.k / 2 + 8) * self.h.abs() + self.k + 4)

    def drop(self, v):
        return v if self.keep is None else torch.where(self.keep, v * self.scale, 0.0)

    def forward(self, dtype):
        v = self.gamma * self.h + self.beta
        tol = self.gamma.abs() * self.dh + 3 * U * (self.gamma * self.h).abs() + 2 * U * (self.beta.abs() + v.abs())
        return self.drop(v), self.drop(tol) + half_step(self.drop(v), dtype)

    def backward(self, gy, dtype):
        """(gx, dgamma, dbeta) and a bound for each."""
        g = self.drop(gy.double())
        dg = U * g.abs()  # the product with dropout's factor
        a, m, k = self.gamma * g, lambda t: t.mean(-1, keepdim=True), self.k
        da = U * 2 * a.abs()
        c1, c2 = m(a), m(a * self.h)
        dc1 = (k + 4) * U * m(a.abs())
        dc2 = (k + 6) * U * m((a * self.h).abs()) + m(a.abs() * self.dh)
        gx = self.s * (a - c1 - self.h * c2)
        # the root's reciprocal is off by (k + 4) / 2 + 3 roundings, the products and differences by one each
        tol = self.s * (da + dc1 + self.dh * c2.abs() + self.h.abs() * dc2 + 4 * U * (a.abs() + c1.abs() + (self.h * c2).abs()))
        tol = tol + gx.abs() * (k / 2 + 6) * U + half_step(gx, dtype)
        n = self.x.shape[0]
        # n terms in any order: n - 1 roundings of the sum of their sizes, and each term's own
        tg = (g.abs() * self.dh + dg * self.h.abs()).sum(0) + (n + 2) * U * (g * self.h).abs().sum(0)
        tb = dg.sum(0) + (n + 2) * U * g.abs().sum(0)
        return (gx, (g * self.h).sum(0), g.sum(0)), (tol, tg + 1e-30, tb + 1e-30)


def assert_within(got, ref, tol, what):
    err = (got.double() - ref).abs()
    bad = ~(err <= tol)
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float((err / tol).nan_to_num(nan=9e9).max()):.3g} of the bound"

"""Plain 64-bit references of the source stack in 8 and 4 bits, and bounds of the
fp32 kernels' rounding errors, derived from the order-free error analysis of
their sums (u = 2^-24, one rounding is at most u; a sum of n products is off by
at most n u of the sum of magnitudes).

Written from the format's definition: codes by search among the magnitudes, the
scale by search among the powers of two.
"""
import numpy as np

U = 2.0 ** -24
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}   # one rounding to the storage
TINY = {"f32": 2.0 ** -150, "bf16": 2.0 ** -134}  # and below its normal numbers
BLOCK = 32
FMTS = ("fp8", "fp4")


def magnitudes(fmt):
    if fmt == "fp4":
        return np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
    m = [k * 2.0 ** -9 for k in range(8)]
    m += [(8 + k) * 2.0 ** (e - 10) for e in range(1, 16) for k in range(8)]
    return np.array(m[:-1])  # the last pattern stands for NaN


def blocks(x):
    d = x.shape[-1]
    pad = -d % BLOCK
    x = np.concatenate([x, np.zeros(x.shape[:-1] + (pad,), x.dtype)], -1)
    return x.reshape(*x.shape[:-1], (d + pad) // BLOCK, BLOCK)


def quantise(x, fmt):
    """(codes, scales) as bytes of x [..., d] in 64 bits."""
    b = blocks(np.asarray(x, np.float64))
    mag = magnitudes(fmt)
    top = np.abs(b).max(-1)
    bad = ~np.isfinite(top)
    limit = mag[-1] * 2.0 ** (np.arange(1, 255) - 127.0)
    e = np.searchsorted(limit, np.where(bad, 0, top)) + 1  # smallest e with top <= limit
    y = np.abs(np.where(bad[..., None], 0, b)) * 2.0 ** (127.0 - e)[..., None]
    hi = np.minimum(np.searchsorted(mag, y), len(mag) - 1)
    lo = np.maximum(hi - 1, 0)
    up, down = mag[hi] - y, y - mag[lo]
    c = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    sign = np.signbit(np.where(bad[..., None], 0, b))
    if fmt == "fp8":
        codes = (c + 128 * sign).astype(np.uint8)
    else:
        c = c + 8 * sign
        codes = (c[..., 0::2] + 16 * c[..., 1::2]).astype(np.uint8)
    return codes.reshape(*x.shape[:-1], codes.shape[-1] * codes.shape[-2]), np.where(bad, 255, e).astype(np.uint8)


def values(codes, scales, d, fmt):
    """The stored values [..., d] in 64 bits."""
    c = codes.astype(np.int64)
    if fmt == "fp4":
        c = np.stack([c % 16, c // 16], -1).reshape(*codes.shape[:-1], 2 * codes.shape[-1])
    half = 128 if fmt == "fp8" else 8
    mag = np.append(magnitudes(fmt), np.nan)
    v = mag[c % half] * np.where(c >= half, -1.0, 1.0)
    p = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    v = v.reshape(*scales.shape, BLOCK) * p[..., None]
    return v.reshape(*scales.shape[:-1], BLOCK * scales.shape[-1])[..., :d]


class Site:
    """One read site in 64 bits: V [S,N,d], keys k [S,N,r] and their results
    with the error bound of each, for results stored as `dtype`."""

    def __init__(self, V, K, q, sliced_r, eps, dtype, dH=None):
        self.V, self.dtype = V, dtype
        self.sliced = K is None
        d = V.shape[2]
        k = V[..., d - sliced_r:] if self.sliced else K
        self.r = r = k.shape[2]
        S, q = V.shape[0], np.asarray(q, np.float64)
        self.rho = rho = np.sqrt((k * k).mean(-1) + eps)
        self.s = s = (k * q).sum(-1) / rho
        a = np.exp(s - s.max(0))
        self.alpha = a = a / a.sum(0)
        # rho: r products summed, divided, + eps, the root (half of them count).
        self.e_rho = e_rho = (r / 2 + 4) * U
        # s: r products summed, and 1 / rho.
        mag = (np.abs(k) * np.abs(q)).sum(-1) / rho
        e_s = (r + 2) * U * mag + (e_rho + U) * np.abs(s)
        # alpha: exp of a difference (each score's error, the largest score's, the
        # subtraction's and the function's 2 ulp), the sum's and the quotient's.
        e_s1 = e_s + U * np.abs(s - s.max(0)) + 4 * U
        rel_a = e_s1 + (a * e_s1).sum(0) + (S + 4) * U
        self.rel_a = rel_a
        self.e_s = e_s
        self.k, self.q, self.d = k, q, d
        # The weights of far sources may underflow: an absolute floor.
        self.e_a = rel_a * a + 2.0 ** -126
        if dH is not None:
            self._backward(dH)

    def _stored(self, x, e):
        return x, 2 * (e + HALF[self.dtype] * np.abs(x) + TINY[self.dtype])

    def h(self):
        S = self.V.shape[0]
        x = np.einsum("sn,snd->nd", self.alpha, self.V)
        mag = np.einsum("sn,snd->nd", self.alpha, np.abs(self.V))
        e = np.einsum("sn,snd->nd", self.e_a, np.abs(self.V)) + (S + 4) * U * mag
        return self._stored(x, e)

    def _backward(self, dH):
        a, V, S = self.alpha, self.V, self.V.shape[0]
        self.dH = dH
        g = (V * dH).sum(-1)
        e_g = (self.d + 2) * U * (np.abs(V) * np.abs(dH)).sum(-1)
        gb = (a * g).sum(0)
        e_gb = (a * e_g + self.e_a * np.abs(g)).sum(0) + (S + 2) * U * (a * np.abs(g)).sum(0)
        self.ds = a * (g - gb)
        diff = np.abs(g - gb)
        self.e_ds = self.e_a * diff + a * (e_g + e_gb + 2 * U * diff)
        self.kbar = self.k / self.rho[..., None]
        self.cq = self.ds / self.rho
        self.e_cq = self.e_ds / self.rho + (self.e_rho + 3 * U) * np.abs(self.cq)
        self.ck = self.cq * self.s / self.r
        self.e_ck = (self.e_cq * np.abs(self.s) + np.abs(self.cq) * (self.e_s + 3 * U * np.abs(self.s))) / self.r

    def coef(self):
        """alpha, ds / rho, ds s / (rho r): [S, 3, N]."""
        x = np.stack([self.alpha, self.cq, self.ck], 1)
        e = np.stack([self.e_a, self.e_cq, self.e_ck], 1)
        return x, 2 * (e + 2 * U * np.abs(x) + 2.0 ** -126)

    def _key_grad(self):
        q, kbar = np.abs(self.q), np.abs(self.kbar)
        x = self.cq[..., None] * self.q - self.ck[..., None] * self.kbar
        e = (self.e_cq[..., None] * q + self.e_ck[..., None] * kbar
             + (self.e_rho + 4 * U) * (np.abs(self.cq)[..., None] * q + np.abs(self.ck)[..., None] * kbar))
        return x, e

    def dV(self, old=None):
        x = self.alpha[..., None] * self.dH
        e = (self.e_a[..., None] + U * self.alpha[..., None]) * np.abs(self.dH)
        if self.sliced:
            y, ey = self._key_grad()
            x[..., self.d - self.r:] += y
            e[..., self.d - self.r:] += ey + 2 * U * np.abs(y)
        return self._sum(x, e, old)

    def dK(self, old=None):
        x, e = self._key_grad()
        return self._sum(x, e, old)

    def _sum(self, x, e, old):
        if old is not None:
            e = e + U * (np.abs(old) + np.abs(x))
            x = x + old
        return self._stored(x, e)

    def dq(self, old=None):
        S, N = self.ds.shape
        t = self.ds[..., None] * self.kbar
        x = t.sum((0, 1))
        mag = np.abs(t).sum((0, 1))
        e = ((self.e_ds[..., None] * np.abs(self.kbar)).sum((0, 1))
             + (self.e_rho + 4 * U + (S * N + 16) * U) * mag)
        if old is not None:
            e, x = e + U * (np.abs(old) + np.abs(x)), x + old
        return x, 2 * (e + U * np.abs(x) + 2.0 ** -126)


def check(name, got, want):
    """Every element within its bound (and nothing but the bound's finite values)."""
    x, bar = want
    got = np.asarray(got, np.float64)
    assert got.shape == x.shape, (name, got.shape, x.shape)
    assert np.isfinite(got).all(), f"{name}: non-finite values"
    worst = (np.abs(got - x) / bar).max(initial=0.0)
    assert worst <= 1.0, f"{name}: error / bound {worst:.3f}"

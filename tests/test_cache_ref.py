"""The references of the 8- and 4-bit source stack, on the CPU: the format against
its definition, the routing of Site against the oracle, its gradients against
central differences, and its error bounds against an fp32 evaluation."""
import numpy as np
import pytest

import oracle
from cache_ref import FMTS, Site, check, magnitudes, quantise, values

EPS = np.float64(np.float32(1e-6))


@pytest.mark.parametrize("fmt", FMTS)
def test_codes_stand_for_themselves(fmt):
    """Every value that a block can hold, beside the largest code, comes back."""
    mag = magnitudes(fmt)
    for e in (1, 2, 100, 127, 200, 246):
        x = np.concatenate([mag, -mag]) * 2.0 ** (e - 127)
        x = x.reshape(-1, 1) * np.ones((1, 2))
        x[:, 1] = mag[-1] * 2.0 ** (e - 127)
        codes, scales = quantise(x, fmt)
        assert (scales == e).all()
        assert np.array_equal(values(codes, scales, 2, fmt), x)


@pytest.mark.parametrize("fmt", FMTS)
def test_rounding_is_nearest(fmt):
    rng = np.random.default_rng(0)
    x = rng.standard_normal((50, 70)) * np.exp(rng.standard_normal((50, 70)))
    codes, scales = quantise(x, fmt)
    y = values(codes, scales, 70, fmt)
    step = 2.0 ** (scales.astype(float) - 127).repeat(32, -1)[:, :70]
    mag = np.concatenate([-magnitudes(fmt)[::-1], magnitudes(fmt)])
    best = np.abs(x[..., None] - mag * step[..., None]).min(-1)
    assert np.array_equal(np.abs(x - y), best)
    # No saturation, and no smaller power of two would do.
    top = np.abs(np.concatenate([x, np.zeros((50, 26))], 1).reshape(50, 3, 32)).max(-1)
    limit = magnitudes(fmt)[-1] * 2.0 ** (scales.astype(float) - 127)
    assert (top <= limit).all() and (top > limit / 2).all()


def problem(seed, S, N, d, r, proj):
    rng = np.random.default_rng(seed)
    V = rng.standard_normal((S, N, d))
    K = rng.standard_normal((S, N, r)) if proj else None
    return V, K, rng.standard_normal(r).astype(np.float32), rng.standard_normal((N, d))


SHAPES = [(1, 3, 40, 8, True), (6, 5, 33, 7, False), (9, 4, 64, 64, False), (17, 2, 50, 24, True)]


@pytest.mark.parametrize("S,N,d,r,proj", SHAPES)
def test_site_matches_the_oracle(S, N, d, r, proj):
    V, K, q, dH = problem(S, S, N, d, r, proj)
    V, dH = V.astype(np.float32), dH.astype(np.float32)
    K = None if K is None else K.astype(np.float32)
    mode = oracle.PROJECTED if proj else oracle.SLICED
    f = lambda x: None if x is None else x.astype(np.float64)  # noqa: E731
    site = Site(f(V), f(K), q, r, EPS, "f32", f(dH))
    np.testing.assert_allclose(site.h()[0], oracle.route_fwd(V, K, q, mode, r=r), rtol=1e-11, atol=1e-12)
    dV, dK, dq = oracle.route_bwd(V, K, q, dH, mode, r=r)
    np.testing.assert_allclose(site.dV()[0] if proj else site.dV()[0], dV, rtol=1e-10, atol=1e-11)
    if proj:
        np.testing.assert_allclose(site.dK()[0], dK, rtol=1e-10, atol=1e-11)
    np.testing.assert_allclose(site.dq()[0], dq, rtol=1e-10, atol=1e-11)


@pytest.mark.parametrize("S,N,d,r,proj", SHAPES)
def test_gradients_match_differences(S, N, d, r, proj):
    V, K, q, dH = problem(S + 50, S, N, d, r, proj)
    rng = np.random.default_rng(1)
    site = Site(V, K, q, r, EPS, "f32", dH)
    pV, pq = rng.standard_normal(V.shape), rng.standard_normal(r)
    pK = None if K is None else rng.standard_normal(K.shape)
    t = 1e-5

    def loss(sign):
        k = None if K is None else K + sign * t * pK
        return (Site(V + sign * t * pV, k, q + sign * t * pq, r, EPS, "f32").h()[0] * dH).sum()

    want = (site.dV()[0] * pV).sum() + (site.dq()[0] * pq).sum()
    if proj:
        want += (site.dK()[0] * pK).sum()
    # Central differences in 64 bits: t^2 terms of about 1e-10 and 2^-53 / t of
    # the loss's size, 1e-10.
    assert abs((loss(1) - loss(-1)) / (2 * t) - want) <= 1e-7 * (1 + np.abs(dH).sum())


@pytest.mark.parametrize("S,N,d,r,proj", SHAPES)
def test_bounds_hold_an_fp32_evaluation(S, N, d, r, proj):
    """Straightforward fp32 arithmetic stays within the bounds, and a perturbed
    query or one swapped source does not."""
    V, K, q, dH = problem(S + 9, S, N, d, r, proj)
    f32 = lambda x: None if x is None else x.astype(np.float32)  # noqa: E731
    V, K, dH = (None if x is None else f32(x).astype(np.float64) for x in (V, K, dH))
    site = Site(V, K, q, r, EPS, "f32", dH)
    v, k, g = f32(V), f32(K), f32(dH)
    k = v[..., d - r:] if k is None else k
    rho = np.sqrt((k * k).sum(-1) / np.float32(r) + np.float32(1e-6))
    s = (k * q).sum(-1) / rho
    a = np.exp(s - s.max(0))
    a = a / a.sum(0)
    h = (a[..., None] * v).sum(0)
    assert h.dtype == np.float32
    check("h", h, site.h())
    ds = a * ((v * g).sum(-1) - (a * (v * g).sum(-1)).sum(0))
    kbar = k / rho[..., None]
    check("dq", (ds[..., None] * kbar).sum((0, 1)), site.dq())
    check("coef", np.stack([a, ds / rho, ds * s / (rho * np.float32(r))], 1), site.coef())
    if S > 1:
        with pytest.raises(AssertionError):
            check("h", (a[::-1, :, None] * v).sum(0), site.h())
        with pytest.raises(AssertionError):
            check("dq", (ds[..., None] * kbar).sum((0, 1)) * np.float32(1.01), site.dq())

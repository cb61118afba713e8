"""The 8- and 4-bit stack on the GPU, as the sizes of real passes reach it: several
tokens a group of lanes at every number of lanes, the most sources there; roundings to
bf16 held to half a step; scores and dots held to what is left where their sums are
exact."""
import numpy as np
import pytest

import paper_2607_09694_amd as lr
from cache_ref import HALF, TINY, U, Site, check, values
from test_gpu_cache import DT, EPS, Problem, check_grads, filled, host, stored

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch.device("cuda:0")


# Several tokens a group start at 8192 tokens for rows of 64 lanes, 16384 for 32 (d
# 257..512 in 8 bits, 513..1024 in 4), 32768 for 16 (16384 forward).
MANY = [
    ("projected", "fp4", 2, 16387, 520, 16), ("sliced", "fp4", 2, 16389, 700, 24),
    ("projected", "fp8", 2, 16387, 300, 16), ("sliced", "fp8", 2, 16385, 500, 13),
    ("projected", "fp8", 2, 8193, 600, 16), ("projected", "fp8", 3, 8197, 1030, 16),
    ("projected", "fp4", 3, 8197, 1030, 16), ("projected", "fp4", 1, 8194, 2050, 8),
    ("projected", "fp8", 1, 4100, 2050, 8), ("sliced", "fp4", 3, 32770, 40, 9),
    ("sliced", "fp8", 5, 32771, 24, 9),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("mode,fmt,S,N,d,r", MANY, ids=[f"{m}_{f}_{S}x{N}x{d}" for m, f, S, N, d, r in MANY])
def test_many_tokens(dev, mode, fmt, S, N, d, r, dtype):
    p = Problem(dev, mode, fmt, dtype, S, N, d, r)
    site = p.site()
    check("h", host(p.fwd()), site.h())
    check_grads(p, p.bwd(), site)
    coef, dq = p.deferred()
    check("coef", host(coef), site.coef())
    check("dq", host(dq), site.dq())


# The most sources of those kernels, whose statistics fill the most on-chip memory.
MOST = [("projected", "fp8", 128, 32771, 200, 16), ("sliced", "fp4", 127, 32769, 96, 96),
        ("projected", "fp8", 128, 16390, 260, 16), ("sliced", "fp4", 127, 16389, 520, 256),
        ("projected", "fp8", 128, 8195, 1030, 256), ("sliced", "fp8", 128, 8196, 560, 33),
        ("projected", "fp4", 129, 16388, 520, 16)]


@pytest.mark.parametrize("mode,fmt,S,N,d,r", MOST, ids=[f"{m}_{f}_{S}x{N}x{d}" for m, f, S, N, d, r in MOST])
def test_many_tokens_of_the_most_sources(dev, mode, fmt, S, N, d, r):
    """Sampled tokens of every kind of place in a wave and a workgroup.  dH is 0 at the
    others, which then add exact zeros to dq."""
    gen = torch.Generator(device=dev).manual_seed(S + N)
    cache = lr.source_cache(S, N, d, fmt, dev)
    cache.codes.random_(0, 256, generator=gen)
    if fmt == "fp8":
        cache.codes.bitwise_and_(0xF7)  # no NaN code
    nb, per = -(-d // 32), 32 if fmt == "fp8" else 16
    past = (nb * 32 - d) * per // 32
    if past:
        cache.codes[..., -past:] = 0
    cache.scales.random_(118, 122, generator=gen)
    q = torch.randn(r, generator=gen, device=dev) / r ** 0.5
    K = torch.randn(S, N, r, generator=gen, device=dev).bfloat16() if mode == "projected" else None
    pick = torch.tensor([0, 1, 2, 3, 7, 15, 16, 31, 64, N // 2, N // 2 + 1, N - 5, N - 2, N - 1], device=dev)
    dH = torch.zeros(N, d, device=dev, dtype=torch.bfloat16)
    dH[pick] = torch.randn(len(pick), d, generator=gen, device=dev).bfloat16()
    print(f"case {mode} {fmt} S={S} N={N} d={d} r={r}", flush=True)
    h = lr.cache_route_fwd(cache, K, q, mode)
    dV, dK, dq = lr.cache_route_bwd(cache, K, q, dH, mode)
    coef = torch.empty((S, 3, N), device=dev)
    dq2 = lr.cache_route_bwd_deferred(cache, K, q, dH, mode, coef)
    torch.cuda.synchronize()
    V = values(cache.codes[:, pick].cpu().numpy(), cache.scales[:, pick].cpu().numpy(), d, fmt)
    site = Site(V, None if K is None else host(K[:, pick]), host(q), r, EPS, "bf16", host(dH[pick]))
    check("h", host(h[pick]), site.h())
    check("dV", host(dV[:, pick]), site.dV())
    if K is not None:
        check("dK", host(dK[:, pick]), site.dK())
    check("dq", host(dq), site.dq())
    check("coef", host(coef[..., pick]), site.coef())
    check("deferred dq", host(dq2), site.dq())


class Tight(Site):
    """Bounds with one rounding to the storage, of half a step: what is stored is a
    number y within 2 e of x, rounded, |y| <= |x| + 2 e."""

    def _stored(self, x, e):
        return x, 2 * e + HALF[self.dtype] * (np.abs(x) + 2 * e) + TINY[self.dtype]


ROUND = [("projected", 9, 7, 100, 24), ("projected", 13, 70, 1000, 50), ("projected", 5, 2053, 64, 8),
         ("sliced", 10, 4, 512, 64), ("sliced", 4, 2051, 100, 19), ("full", 7, 5, 50, 50),
         ("full", 11, 9, 512, 512), ("full", 6, 4, 1100, 1100), ("full", 4, 2061, 72, 72)]


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
@pytest.mark.parametrize("mode,S,N,d,r", ROUND, ids=[f"{m}_{S}x{N}x{d}" for m, S, N, d, r in ROUND])
def test_bf16_results_round_to_nearest(dev, mode, S, N, d, r, fmt):
    p = Problem(dev, mode, fmt, "bf16", S, N, d, r)
    site = p.site()
    site.__class__ = Tight
    check("h", host(p.fwd()), site.h())
    check_grads(p, p.bwd(), site)
    rng = np.random.default_rng(3)
    dV, oV = stored(rng.standard_normal((S, N, d)), "bf16", dev)
    dK, oK = stored(rng.standard_normal((S, N, r)), "bf16", dev) if mode == "projected" else (None, None)
    dq, oq = stored(rng.standard_normal(p.r), "f32", dev)
    got = p.bwd(out=(dV, dK, dq), accumulate=True)
    check_grads(p, got, site, (oV, oK, oq))


class ExactScores(Site):
    """Bounds where q . k is exact in fp32: what is left of a score is 1 / rho and its
    product."""

    def __init__(self, V, K, q, r, dtype, dH):
        super().__init__(V, K, q, r, EPS, dtype)
        self.e_s = (self.e_rho + 3 * U) * np.abs(self.s)
        e_s1 = self.e_s + U * np.abs(self.s - self.s.max(0)) + 4 * U
        self.rel_a = e_s1 + (self.alpha * e_s1).sum(0) + (V.shape[0] + 4) * U
        self.e_a = self.rel_a * self.alpha + 2.0 ** -126
        self._backward(dH)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
@pytest.mark.parametrize("mode,S,N,d", [("full", 5, 6, 96), ("full", 20, 3, 1024), ("full", 3, 2100, 160),
                                        ("full", 9, 2, 1500), ("sliced", 5, 6, 96), ("sliced", 3, 1100, 160),
                                        ("projected", 5, 6, 96), ("projected", 3, 1100, 96)])
def test_cancelling_scores(dev, mode, S, N, d, fmt, dtype):
    """A query whose parts of 20 bits cancel but for a thousandth: columns a and b of
    every key are equal and meet q_a = -q_b + a small part.  Products are multiples of
    2^-15 whose magnitudes sum to less than 2^24 of these, so q . k is exact in any order;
    a query held to 16 bits would be off by 1e-3 in the scores."""
    rng = np.random.default_rng(S + d)
    r = d
    grid = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
    q = np.zeros(r)
    pairs = ((3, r - 7), (40, r // 2 + 5))
    for a, b in pairs:
        q[a] = rng.integers(1_000_000, 1_250_000) * 2.0 ** -14
        q[b] = -q[a] + rng.integers(8_000, 16_000) * 2.0 ** -14

    def rows():
        x = grid[rng.integers(0, 8, (S, N, d))] * rng.choice([-1.0, 1.0], (S, N, d))
        x[..., 0::32] = 6.0  # every block's scale is 2^0 (e4m3: exact too)
        for a, b in pairs:
            x[..., a] = x[..., b] = grid[rng.integers(1, 4, (S, N))] * rng.choice([-1.0, 1.0], (S, N))
        return x

    V, K, k = rows(), None, None
    if mode == "projected":
        K, k = stored(rows(), dtype, dev)
    cache, stack = filled(V, fmt, dev)
    assert np.array_equal(stack, V)
    keys = stack if k is None else k
    assert ((np.abs(keys) * np.abs(q)).sum(-1) < 2.0 ** 24 * 2.0 ** -15).all()
    dH, dh = stored(rng.standard_normal((N, d)), dtype, dev)
    qt = torch.from_numpy(q.astype(np.float32)).to(dev)
    print(f"case {mode} {fmt} {dtype} S={S} N={N} d={d}", flush=True)
    site = ExactScores(stack, k, q, r, dtype, dh)
    check("h", host(lr.cache_route_fwd(cache, K, qt, mode, dtype=DT[dtype])), site.h())
    dV, dK, dq = lr.cache_route_bwd(cache, K, qt, dH, mode)
    check("dV", host(dV), site.dV())
    if K is not None:
        check("dK", host(dK), site.dK())
    check("dq", host(dq), site.dq())


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
@pytest.mark.parametrize("mode", ["projected", "sliced", "full"])
@pytest.mark.parametrize("S,N,bad", [(8, 3, (0, 1)), (8, 3, (6, 7)), (9, 2, (2, 3, 4, 5, 6, 7, 8)),
                                     (5, 1100, (0, 1, 2)), (64, 2, tuple(range(16)))])
def test_scores_below_the_range(dev, mode, S, N, bad, fmt):
    """q . k of a few sources is below fp32's range (-inf): they weigh nothing beside the
    others, however a token's sources are split."""
    rng = np.random.default_rng(S)
    d = r = 64
    V = rng.standard_normal((S, N, d))
    K = k = None
    q = rng.standard_normal(r) / 8
    q[0] = 2.0 ** 90
    keys = V
    if mode == "projected":
        keys = rng.standard_normal((S, N, r))
    keys[..., :32] = 0.0
    keys[list(bad), :, 0] = -2.0 ** 55  # |k|^2 and rho are in range
    if mode == "projected":
        K, k = stored(keys, "f32", dev)
    cache, stack = filled(V, fmt, dev)
    h = lr.cache_route_fwd(cache, K, torch.from_numpy(q.astype(np.float32)).to(dev), mode, dtype=torch.float32)
    check("h", host(h), Site(stack, k, q.astype(np.float32), r, EPS, "f32").h())

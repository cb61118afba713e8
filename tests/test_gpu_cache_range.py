"""Full-rank backward over the 4-bit stack where a block of 32 columns of q or dH
has range: a column far larger than the others must not cost the others their fp32
accuracy, whatever the rows hold there.  Bounds are those of fp32 arithmetic
(tests/cache_ref.py) or, where every sum is a whole number of granules below 2^24,
of the few roundings that remain."""
import numpy as np
import pytest

import paper_2607_09694_amd as lr
from cache_ref import BLOCK, U, Site, check
from test_gpu_cache import EPS, check_grads, filled, host, stored

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch.device("cuda:0")


class Full:
    """One full-rank site: rows V (quantised here), q and dH as given."""

    def __init__(self, dev, fmt, dtype, V, q, dH):
        self.cache, self.V = filled(V, fmt, dev)
        self.q = torch.from_numpy(np.asarray(q, np.float32)).to(dev)
        self.dH, self.dh = stored(dH, dtype, dev)
        self.mode, self.dtype, self.r = "full", dtype, V.shape[2]
        print(f"case full {fmt} {dtype} {V.shape}", flush=True)

    def site(self):
        return Site(self.V, None, host(self.q), self.r, EPS, self.dtype, self.dh)

    def bwd(self):
        got = lr.cache_route_bwd(self.cache, None, self.q, self.dH, "full")
        torch.cuda.synchronize()
        return got


# Sources of one tile and of several, tokens that share a workgroup, rows of part of a
# block, of one and of several column chunks.
SHAPES = [(4, 5, 64), (17, 4, 1024), (33, 3, 2047), (5, 2100, 96), (2, 3, 33), (9, 1, 4096)]


@pytest.mark.parametrize("where", ["dH", "q", "both"])
@pytest.mark.parametrize("size", [1e2, 1e5, 1e9])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
@pytest.mark.parametrize("S,N,d", SHAPES, ids=[f"{S}x{N}x{d}" for S, N, d in SHAPES])
def test_outlier_columns(dev, S, N, d, fmt, dtype, size, where):
    """One column of every block is far larger in dH or q, and its codes are 0 (the
    column is 2^-24 of its neighbours): it has no part in any dot."""
    rng = np.random.default_rng(1000 * S + d)
    V, dH = rng.standard_normal((S, N, d)), rng.standard_normal((N, d))
    q = rng.standard_normal(d) / np.sqrt(d)
    V[..., 5::BLOCK] *= 2.0 ** -24
    if where != "q":
        dH[:, 5::BLOCK] *= size
    if where != "dH":
        q[5::BLOCK] *= size
    p = Full(dev, fmt, dtype, V, q, dH)
    check_grads(p, p.bwd(), p.site())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
@pytest.mark.parametrize("S,N,d", [(2, 3, 256), (16, 2, 1024), (32, 3, 2048), (4, 2100, 128)])
def test_exact_dots(dev, S, N, d, fmt, dtype):
    """q = 0, so that every weight is 1 / S exactly, and rows and dH of small whole
    numbers: dH . x, its mean over the sources and ds are exact in fp32 in any order,
    whatever the blocks' scales (2^0 to 2^20 within 128 columns) and whatever dH holds
    where the rows are 0 (2^30).  What is left of dq is 1 / rho, its product with the
    code and the products' sum.

    Every product is a multiple of 1/2 and their magnitudes sum to less than 2^24 of
    these, so no partial sum rounds."""
    rng = np.random.default_rng(d + S)
    V = np.zeros((S, N, d))
    dH = np.zeros((N, d))
    cols = np.arange(d)
    small = cols % 128 < 64
    V[..., small] = rng.integers(-6, 7, (S, N, small.sum()))
    V[..., 0::BLOCK] = 6.0  # every block's scale: 6 is the largest code, or exact in e4m3
    dH[:, small] = rng.integers(-3, 4, (N, small.sum()))
    V[..., 5::BLOCK] = 0.0
    dH[:, 5::BLOCK] = 2.0 ** 30
    for c in (70, 128 * (d // 128) - 20):  # a block each of far larger scale
        b = c // BLOCK * BLOCK
        V[..., b:b + BLOCK] = 0.0
        V[..., c] = 2.0 ** 20
        dH[:, b:b + BLOCK] = 0.0
        dH[:, c] = 1.0 if c == 70 else -1.0
    p = Full(dev, fmt, dtype, V, np.zeros(d), dH)
    site = p.site()
    # Whole numbers in e2m1 round to codes 0 .. 6: p.V holds what is stored.
    assert (np.abs(p.V).max(-1) == 2.0 ** 20).all()
    assert (2 * np.abs(p.dh * p.V).sum(-1) < 2 ** 24).all()
    assert np.array_equal(site.alpha, np.full((S, N), 1 / S))
    got = p.bwd()
    check("dV", host(got[0]), site._stored(site.alpha[..., None] * p.dh, 2 * U * np.abs(p.dh)))
    t = np.abs(site.ds[..., None] * site.kbar).sum((0, 1))
    x, _ = site.dq()
    check("dq", host(got[2]), (x, 2 * (site.e_rho + (S * N + 16) * U) * t + 2.0 ** -120))


@pytest.mark.parametrize("S,N,d", [(3, 2, 64), (20, 3, 300)])
def test_tiny_and_large_scales(dev, S, N, d):
    """Rows at and below the smallest normal number (codes of 1/2 at 2^-126) against a
    large dH, and large rows against a small one."""
    rng = np.random.default_rng(9)
    for v, g in ((2.0 ** -125, 2.0 ** 117), (2.0 ** 30, 2.0 ** -60)):
        V, dH = v * rng.standard_normal((S, N, d)), g * rng.standard_normal((N, d))
        p = Full(dev, "fp4", "f32", V, rng.standard_normal(d), dH)
        site = p.site()
        dV, dK, dq = p.bwd()
        # |x|^2 of the tiny rows underflows beside eps, as its bound says.  dV's factor of
        # x, ds s / (rho^2 d), is an fp32 number: where the weights leave 2^-126 it is off
        # by half of its smallest step, 2^-150, and dV by that times |x| (twice, as all
        # bounds are).
        x, e = site.dV()
        check("dV", host(dV), (x, e + 2.0 ** -149 * np.abs(p.V)))
        check("dq", host(dq), site.dq())
        assert dK is None


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
def test_largest_finite_gradient(dev, fmt, dtype):
    """A dH near the largest number of its type counts as what it is: finite where the
    rows are 0."""
    rng = np.random.default_rng(4)
    S, N, d = 6, 4, 96
    V, dH = rng.standard_normal((S, N, d)), rng.standard_normal((N, d))
    V[..., 40] = 0.0
    dH[1, 40] = 3.3e38
    p = Full(dev, fmt, dtype, V, rng.standard_normal(d) / 10, dH)
    check_grads(p, p.bwd(), p.site())


def test_most_sources_of_the_widest_matrix_rows(dev):
    """The most on-chip memory that rows of up to 1024 columns take."""
    rng = np.random.default_rng(6)
    S, N, d = 512, 2, 1024
    V, dH = rng.standard_normal((S, N, d)), rng.standard_normal((N, d))
    p = Full(dev, "fp4", "f32", V, rng.standard_normal(d) / 32, dH)
    check_grads(p, p.bwd(), p.site())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("fmt,first", [("fp8", 1 - 2.0 ** -5), ("fp4", 1 - 2.0 ** -3)])
def test_sources_that_round_to_two_to_the_128(dev, fmt, first, dtype):
    """The largest sources: those that round to 2^128 read as infinities, the one before
    them as the code below."""
    step = 2.0 ** (-24 if dtype == "f32" else -8)
    x = np.full((1, 2, 64), 1.0)
    x[0, 0, 3], x[0, 0, 40] = first * 2.0 ** 127 * 2, -(first - step) * 2.0 ** 127 * 2
    x[0, 1, 9] = (first - step) * 2.0 ** 127 * 2
    O, exact = stored(x, dtype, dev)
    assert np.array_equal(exact, x)  # every input is a number of the storage
    cache = lr.source_cache(1, 2, 64, fmt, dev)
    lr.cache_write(cache, O)
    got = host(lr.cache_read(cache, O.dtype))
    below = (1 - 2.0 ** -4) * 2.0 ** 127 * 2 if fmt == "fp8" else 0.75 * 2.0 ** 127 * 2
    assert got[0, 0, 3] == np.inf and got[0, 0, 40] == -below and got[0, 1, 9] == below
    assert np.isfinite(np.delete(got.reshape(-1), 3)).all()

"""The source stack in 8 and 4 bits on the GPU: the format bit for bit, and the
routing over it, forward and backward, within the error bounds of its fp32
arithmetic (tests/cache_ref.py), at the sizes and values where it can go wrong."""
import numpy as np
import pytest

import paper_2607_09694_amd as lr
from cache_ref import BLOCK, FMTS, Site, check, magnitudes, quantise, values

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
EPS = np.float64(np.float32(1e-6))
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch.device("cuda:0")


def host(t):
    return t.detach().double().cpu().numpy()


def stored(x, dtype, dev):
    """x rounded to the storage on the GPU, and those values in 64 bits."""
    t = torch.from_numpy(np.asarray(x, np.float32)).to(dev).to(DT[dtype])
    return t, host(t)


def filled(V, fmt, dev):
    """A cache that holds V's quantised values, and those values in 64 bits."""
    codes, scales = quantise(V, fmt)
    d = V.shape[-1]
    c = lr.SourceCache(torch.from_numpy(codes).to(dev), torch.from_numpy(scales).to(dev), d, fmt)
    return c, values(codes, scales, d, fmt)


class Problem:
    def __init__(self, dev, mode, fmt, dtype, S, N, d, r, seed=0, spread=0.5):
        rng = np.random.default_rng(seed + 1000 * S + N + d)
        V = rng.standard_normal((S, N, d)) * np.exp(spread * rng.standard_normal((1, 1, d)))
        self.cache, self.V = filled(V, fmt, dev)
        self.K = self.k = None
        if mode == "projected":
            self.K, self.k = stored(rng.standard_normal((S, N, r)), dtype, dev)
        self.r = d if mode == "full" else r
        self.q = torch.from_numpy((rng.standard_normal(self.r) / np.sqrt(self.r)).astype(np.float32)).to(dev)
        self.dH, self.dh = stored(rng.standard_normal((N, d)), dtype, dev)
        self.mode, self.fmt, self.dtype = mode, fmt, dtype
        print(f"case {mode} {fmt} {dtype} S={S} N={N} d={d} r={r}", flush=True)

    def site(self, grad=True):
        return Site(self.V, self.k, host(self.q), self.r, EPS, self.dtype, self.dh if grad else None)

    def fwd(self, **kw):
        return lr.cache_route_fwd(self.cache, self.K, self.q, self.mode, dtype=DT[self.dtype], **kw)

    def bwd(self, **kw):
        return lr.cache_route_bwd(self.cache, self.K, self.q, self.dH, self.mode, **kw)

    def deferred(self, **kw):
        S, N, _ = self.cache.shape
        coef = torch.full((S, 3, N), float("nan"), device=self.q.device)
        return coef, lr.cache_route_bwd_deferred(self.cache, self.K, self.q, self.dH, self.mode,
                                                 coef, **kw)


def check_grads(p, got, site, old=(None, None, None)):
    dV, dK, dq = got
    check("dV", host(dV), site.dV(old[0]))
    if p.mode == "projected":
        check("dK", host(dK), site.dK(old[1]))
    else:
        assert dK is None
    check("dq", host(dq), site.dq(old[2]))


# ---------------------------------------------------------------------------
# Writing and reading
# ---------------------------------------------------------------------------


def special_rows(d, dtype, seed):
    """Rows of ordinary values and of every kind that the format treats apart."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((40, d)) * np.exp(3 * rng.standard_normal((40, 1)))
    x[1] = 0.0
    x[2] = -0.0
    x[3] = rng.standard_normal(d) * 1e-39           # fp32 subnormals
    x[4] = rng.standard_normal(d) * 2.0 ** -125      # smallest scale
    x[5] = np.where(rng.random(d) < 0.5, 3.38e38, -1e36)
    x[6] = 448.0 * np.where(rng.random(d) < 0.5, 1, -1)  # exactly the largest code
    x[7] = 6.0
    x[8] = np.float32(448.0) * (1 + 2.0 ** -7)       # just above it
    x[9, 0] = np.nan
    x[10, -1] = np.inf
    x[11, d // 2] = -np.inf
    x[12, 0], x[12, -1] = -np.nan, np.inf
    # Halfway between neighbouring codes, beside a largest code.
    for k, fmt in ((13, "fp8"), (14, "fp4")):
        m = magnitudes(fmt)
        mid = (m[1:] + m[:-1]) / 2
        x[k] = np.resize(mid, d) * np.where(np.arange(d) % 3 == 0, -1, 1)
        x[k, ::BLOCK] = m[-1]
    x = x.astype(np.float32)
    return x if dtype == "f32" else host(torch.from_numpy(x).bfloat16()).astype(np.float32)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [1, 2, 7, 8, 31, 32, 33, 40, 100, 1000, 1024, 2047, 8200])
def test_write_is_the_format(dev, fmt, dtype, d):
    x = special_rows(d, dtype, d)
    O = torch.from_numpy(x).to(dev).to(DT[dtype])[None].contiguous()
    cache = lr.source_cache(3, 40, d, fmt, dev)
    cache.codes.fill_(0xA5)
    cache.scales.fill_(0x5A)
    lr.cache_write(cache.planes(1), O)
    torch.cuda.synchronize()
    codes, scales = quantise(x, fmt)
    assert np.array_equal(cache.scales[1].cpu().numpy(), scales)
    assert np.array_equal(cache.codes[1].cpu().numpy(), codes)
    for k in (0, 2):  # the planes beside it
        assert (cache.codes[k] == 0xA5).all() and (cache.scales[k] == 0x5A).all()


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_read_every_code_and_scale(dev, fmt, dtype):
    n = 256
    codes = np.arange(n, dtype=np.uint8)
    codes = np.tile(codes, (n, 1))                       # 256 rows of every byte
    per = BLOCK if fmt == "fp8" else BLOCK // 2
    scales = np.repeat(np.arange(n, dtype=np.uint8)[:, None], n // per, 1)
    d = n if fmt == "fp8" else 2 * n
    c = lr.SourceCache(torch.from_numpy(codes[None].copy()).to(dev),
                       torch.from_numpy(scales[None].copy()).to(dev), d, fmt)
    got = lr.cache_read(c, DT[dtype])[0].cpu()
    want = torch.from_numpy(values(codes, scales, d, fmt)).to(torch.float32).to(DT[dtype])
    assert torch.equal(got.isnan(), want.isnan())
    assert torch.equal(got.nan_to_num(7.0, 1e30, -1e30), want.nan_to_num(7.0, 1e30, -1e30))


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("S,N,d", [(1, 1, 1), (2, 3, 50), (3, 67, 1000), (1, 1300, 24), (2, 5, 4096)])
def test_write_then_read_and_guards(dev, fmt, dtype, S, N, d):
    rng = np.random.default_rng(d)
    O, x = stored(rng.standard_normal((S, N, d)), dtype, dev)
    cache = lr.source_cache(S, N, d, fmt, dev)
    lr.cache_write(cache, O)
    buf = torch.full((S * N * d + 64,), 77.0, dtype=DT[dtype], device=dev)
    out = buf[32:32 + S * N * d].view(S, N, d)
    assert lr.cache_read(cache, out=out) is out
    want = values(*quantise(x, fmt), d, fmt)
    assert np.array_equal(host(out), want)
    assert (buf[:32] == 77).all() and (buf[-32:] == 77).all()


@pytest.mark.parametrize("fmt", FMTS)
def test_odd_element_addresses(dev, fmt):
    """Rows whose base is not 16-byte aligned go element by element, same bits."""
    rng = np.random.default_rng(5)
    flat = torch.from_numpy(rng.standard_normal(1 + 6 * 64).astype(np.float32)).to(dev).bfloat16()
    O = flat[1:].view(1, 6, 64)
    a, b = lr.source_cache(1, 6, 64, fmt, dev), lr.source_cache(1, 6, 64, fmt, dev)
    lr.cache_write(a, O)
    lr.cache_write(b, O.clone())
    assert torch.equal(a.codes, b.codes) and torch.equal(a.scales, b.scales)
    out = torch.empty(1 + 6 * 64, dtype=torch.bfloat16, device=dev)
    lr.cache_read(a, out=out[1:].view(1, 6, 64))
    assert torch.equal(out[1:].view(1, 6, 64), lr.cache_read(b))


# ---------------------------------------------------------------------------
# One site
# ---------------------------------------------------------------------------

# (mode, S, N, d, r): one and two sources, few and many of them, one token and
# ragged token groups, rows of part of a block, of whole lanes, of several
# chunks; keys that start inside a lane's columns and inside a block.
SITES = [
    ("projected", 1, 1, 1, 1), ("projected", 2, 3, 33, 5), ("projected", 5, 1, 64, 8),
    ("projected", 9, 7, 100, 24), ("projected", 49, 3, 1024, 16), ("projected", 13, 70, 1000, 50),
    ("projected", 64, 5, 2048, 32), ("projected", 3, 9, 2500, 256), ("projected", 200, 2, 96, 12),
    ("sliced", 1, 2, 1, 1), ("sliced", 2, 3, 33, 33), ("sliced", 7, 5, 50, 13),
    ("sliced", 10, 4, 512, 64), ("sliced", 25, 6, 1024, 128), ("sliced", 33, 3, 1021, 255),
    ("sliced", 6, 11, 2047, 256), ("sliced", 12, 2, 4096, 7), ("sliced", 130, 3, 40, 9),
    ("full", 1, 1, 1, 1), ("full", 2, 3, 33, 33), ("full", 7, 5, 50, 50), ("full", 11, 9, 512, 512),
    ("full", 49, 3, 1024, 1024), ("full", 6, 17, 1021, 1021), ("full", 9, 4, 2048, 2048),
    ("full", 5, 3, 3001, 3001), ("full", 70, 2, 64, 64),
]
# More tokens than are split over workgroups, kept small otherwise.
MANY = [
    ("projected", 5, 2053, 64, 8), ("projected", 3, 2500, 1000, 24), ("projected", 4, 4400, 40, 9),
    ("sliced", 4, 2051, 100, 19), ("sliced", 3, 2100, 1056, 64), ("sliced", 2, 4500, 33, 8),
    ("full", 4, 2061, 72, 72), ("full", 3, 2050, 1040, 1040), ("full", 3, 4200, 31, 31),
    ("projected", 3, 8197, 33, 8), ("sliced", 2, 8203, 1030, 16), ("full", 2, 8195, 40, 40),
    ("projected", 2, 33001, 24, 4), ("sliced", 2, 4099, 2300, 40),
]
IDS = [f"{m}_{S}x{N}x{d}_r{r}" for m, S, N, d, r in SITES + MANY]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("mode,S,N,d,r", SITES + MANY, ids=IDS)
def test_forward(dev, mode, S, N, d, r, fmt, dtype):
    p = Problem(dev, mode, fmt, dtype, S, N, d, r)
    buf = torch.full((N * d + 64,), 77.0, dtype=DT[dtype], device=dev)
    out = buf[32:32 + N * d].view(N, d)
    assert p.fwd(out=out) is out
    torch.cuda.synchronize()
    check("h", host(out), p.site(False).h())
    assert (buf[:32] == 77).all() and (buf[-32:] == 77).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("mode,S,N,d,r", SITES + MANY, ids=IDS)
def test_backward(dev, mode, S, N, d, r, fmt, dtype):
    p = Problem(dev, mode, fmt, dtype, S, N, d, r)
    site = p.site()
    got = p.bwd()
    torch.cuda.synchronize()
    check_grads(p, got, site)


@pytest.mark.parametrize("fmt,dtype", [("fp8", "bf16"), ("fp4", "f32")])
@pytest.mark.parametrize("mode,S,N,d,r", SITES[::2] + MANY[::3], ids=IDS[:len(SITES)][::2] + IDS[len(SITES):][::3])
def test_backward_adds(dev, mode, S, N, d, r, fmt, dtype):
    p = Problem(dev, mode, fmt, dtype, S, N, d, r)
    rng = np.random.default_rng(3)
    dV, oV = stored(rng.standard_normal((S, N, d)), dtype, dev)
    dK, oK = stored(rng.standard_normal((S, N, r)), dtype, dev) if mode == "projected" else (None, None)
    dq, oq = stored(rng.standard_normal(p.r), "f32", dev)
    got = p.bwd(out=(dV, dK, dq), accumulate=True)
    assert got[0] is dV and got[2] is dq
    torch.cuda.synchronize()
    check_grads(p, got, p.site(), (oV, oK, oq))


LOWRANK = [c for c in SITES + MANY if c[0] != "full"]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("mode,S,N,d,r", LOWRANK, ids=[f"{m}_{S}x{N}x{d}_r{r}" for m, S, N, d, r in LOWRANK])
def test_deferred(dev, mode, S, N, d, r, fmt, dtype):
    p = Problem(dev, mode, fmt, dtype, S, N, d, r)
    coef, dq = p.deferred()
    torch.cuda.synchronize()
    site = p.site()
    check("coef", host(coef), site.coef())
    check("dq", host(dq), site.dq())


@pytest.mark.parametrize("d,r", [(4100, 30), (9000, 5000), (10240, 10240)])
def test_wide_forward(dev, d, r):
    """Rows wider than one wave's columns, keys wider than a wave's slots."""
    for N in (3, 2100):
        if N * d > 2100 * 4100:
            N = 5
        p = Problem(dev, "sliced", "fp8", "f32", 4, N, d, r)
        check("h", host(p.fwd()), p.site(False).h())


@pytest.mark.parametrize("fmt", FMTS)
def test_most_on_chip_memory(dev, fmt):
    """The most sources, the widest rows and the narrowest (the most tokens a wave)."""
    for mode, S, N, d, r in (("full", 512, 2, 4096, 4096), ("full", 512, 3, 40, 40),
                             ("sliced", 512, 3, 70, 20), ("projected", 500, 1026, 20, 8)):
        p = Problem(dev, mode, fmt, "f32", S, N, d, r)
        site = p.site()
        check("h", host(p.fwd()), site.h())
        check_grads(p, p.bwd(), site)


def test_most_sources(dev):
    p = Problem(dev, "projected", "fp8", "bf16", 1024, 1030, 16, 4)
    check("h", host(p.fwd()), p.site(False).h())
    p = Problem(dev, "projected", "fp4", "f32", 1024, 2, 64, 8)
    check("h", host(p.fwd()), p.site(False).h())
    p = Problem(dev, "sliced", "fp8", "bf16", 512, 3, 48, 16)
    check_grads(p, p.bwd(), p.site())


# Decoding: the newest source is written by the site that first reads it.
APPEND = [("projected", 1, 1, 64, 8), ("projected", 49, 16, 1024, 16), ("projected", 7, 5, 33, 4),
          ("projected", 3, 2100, 64, 8), ("sliced", 1, 3, 40, 9), ("sliced", 26, 7, 1024, 64),
          ("sliced", 5, 2, 2047, 100), ("sliced", 4, 2100, 50, 13), ("full", 1, 1, 33, 33),
          ("full", 10, 3, 1024, 1024), ("full", 5, 2, 2050, 2050), ("full", 3, 1100, 72, 72),
          ("sliced", 3, 2, 5000, 40)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("mode,S,N,d,r", APPEND, ids=[f"{m}_{S}x{N}x{d}_r{r}" for m, S, N, d, r in APPEND])
def test_newest_source_written_by_its_site(dev, mode, S, N, d, r, fmt, dtype):
    p = Problem(dev, mode, fmt, dtype, S, N, d, r)
    rng = np.random.default_rng(8)
    o, x = stored(rng.standard_normal((N, d)), dtype, dev)
    before = (p.cache.codes[:-1].clone(), p.cache.scales[:-1].clone())
    h = p.fwd(o_new=o)
    torch.cuda.synchronize()
    codes, scales = quantise(x, fmt)
    assert np.array_equal(p.cache.codes[-1].cpu().numpy(), codes)
    assert np.array_equal(p.cache.scales[-1].cpu().numpy(), scales)
    assert torch.equal(p.cache.codes[:-1], before[0]) and torch.equal(p.cache.scales[:-1], before[1])
    p.V[-1] = values(codes, scales, d, fmt)
    check("h", host(h), p.site(False).h())


@pytest.mark.parametrize("mode", ["projected", "sliced", "full"])
def test_no_tokens(dev, mode):
    p = Problem(dev, mode, "fp8", "bf16", 4, 0, 64, 8)
    assert p.fwd().shape == (0, 64)
    dV, dK, dq = p.bwd()
    assert dV.shape == (4, 0, 64) and torch.equal(dq, torch.zeros_like(dq))
    if mode != "full":
        assert torch.equal(p.deferred()[1], torch.zeros_like(dq))
    lr.cache_write(p.cache, torch.empty((4, 0, 64), device=dev))
    assert lr.cache_read(p.cache).shape == (4, 0, 64)


@pytest.mark.parametrize("mode", ["projected", "sliced", "full"])
@pytest.mark.parametrize("N", [6, 2100])
def test_nan_block_stays_with_its_token(dev, mode, N):
    """A block that was written from a NaN or an infinity makes its own token's
    results NaN (full rank and sliced: every weight; projected: its columns)."""
    p = Problem(dev, mode, "fp8", "f32", 5, N, 96, 16)
    clean = p.fwd()
    grads = p.bwd()
    p.cache.scales[2, 1, 2] = 255
    h = p.fwd()
    dV, dK, dq = p.bwd()
    keep = torch.arange(N, device=dev) != 1
    assert torch.equal(h[keep], clean[keep])
    assert torch.equal(dV[:, keep], grads[0][:, keep])
    assert h[1, 64:].isnan().all()
    if mode == "projected":
        assert torch.equal(h[1, :64], clean[1, :64])
    else:
        assert h[1].isnan().all() and dV[:, 1].isnan().any()
    assert dq.isnan().any()  # the sum over tokens


def test_peaked_and_equal_scores(dev):
    """One source takes all the weight; all sources take the same."""
    for scale in (0.0, 300.0):
        for mode in ("projected", "sliced", "full"):
            p = Problem(dev, mode, "fp8", "f32", 11, 9, 64, 16)
            p.q.mul_(scale)
            check("h", host(p.fwd()), p.site(False).h())
            check_grads(p, p.bwd(), p.site())


def test_differences(dev):
    """dq and dK against central differences of the forward kernel itself: with
    step t = 2^-6 the t^2 term (third derivatives of a softmax of scores of size
    about 1, below 1) is within 2^-12 |p|^3, and the difference of two fp32 losses
    is off by at most 2 N d u max|h dH| / t."""
    p = Problem(dev, "projected", "fp8", "f32", 8, 5, 64, 16)
    rng = np.random.default_rng(2)
    _, dK, dq = p.bwd()
    loss = lambda: float((host(p.fwd()) * p.dh).sum())  # noqa: E731
    t = 2.0 ** -6
    for x, grad in ((p.q, dq), (p.K, dK)):
        e = rng.standard_normal(tuple(x.shape))
        e = torch.from_numpy((e / np.linalg.norm(e)).astype(np.float32)).to(dev)
        keep = x.clone()
        x.copy_(keep + t * e)
        up = loss()
        x.copy_(keep - t * e)
        down = loss()
        x.copy_(keep)
        size = np.abs(host(p.fwd()) * p.dh).sum()
        assert abs((up - down) / (2 * t) - float((grad * e).sum())) <= size * (2.0 ** -12 + 4 * 2.0 ** -24 / t)


# ---------------------------------------------------------------------------
# Use
# ---------------------------------------------------------------------------


@pytest.mark.parametrize("mode,N", [("projected", 40), ("sliced", 40), ("full", 40), ("projected", 2100)])
def test_reproducible(dev, mode, N):
    p = Problem(dev, mode, "fp8", "bf16", 17, N, 200, 24)
    a, b = (p.fwd(), *p.bwd()), (p.fwd(), *p.bwd())
    for x, y in zip(a, b):
        assert (x is None and y is None) or torch.equal(x, y)


def test_dirty_workspace_and_outputs(dev):
    p = Problem(dev, "projected", "fp4", "bf16", 12, 70, 300, 24)
    want = p.bwd()
    S, N, d = p.cache.shape
    need = lr.cache_route_bwd_workspace_bytes(S, N, d, 24, "projected", "fp4", torch.bfloat16)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device=dev)
    out = tuple(torch.full_like(x, float("nan")) for x in want)
    got = p.bwd(out=out, workspace=ws)
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    with pytest.raises(lr.RoutingError, match="workspace"):
        p.bwd(workspace=ws[:need - 4])


def test_other_stream(dev):
    p = Problem(dev, "sliced", "fp8", "bf16", 20, 300, 512, 32)
    want = (p.fwd(), *p.bwd())
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        got = (p.fwd(), *p.bwd())
    st.synchronize()
    for x, y in zip(got, want):
        assert (x is None and y is None) or torch.equal(x, y)


def test_two_streams_at_once(dev):
    """Calls in flight together, each with a workspace of its own."""
    ps = [Problem(dev, m, f, "bf16", 30, 900, 520, 24) for m, f in
          (("projected", "fp8"), ("sliced", "fp4"), ("full", "fp4"), ("full", "fp8"))]
    want = [(p.fwd(), *p.bwd()) for p in ps]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in ps]
    got = [None] * len(ps)
    for _ in range(3):
        for k, (p, st) in enumerate(zip(ps, streams)):
            with torch.cuda.stream(st):
                got[k] = (p.fwd(), *p.bwd())
    torch.cuda.synchronize()
    for w, g in zip(want, got):
        for x, y in zip(w, g):
            assert (x is None and y is None) or torch.equal(x, y)


def test_random_shapes(dev):
    """Seeded shapes over the whole range, every call."""
    rng = np.random.default_rng(77)
    for k in range(60):
        mode = ("projected", "sliced", "full")[k % 3]
        fmt, dtype = FMTS[k // 3 % 2], ("bf16", "f32")[k // 6 % 2]
        S = int(np.exp(rng.uniform(0, np.log(70))))
        d = int(np.exp(rng.uniform(0, np.log(2500))))
        N = min(int(np.exp(rng.uniform(0, np.log(9000)))), max(1, 1_500_000 // (S * d)))
        r = min(d, int(np.exp(rng.uniform(0, np.log(256))))) if mode == "sliced" else \
            int(np.exp(rng.uniform(0, np.log(256))))
        p = Problem(dev, mode, fmt, dtype, S, N, d, r, seed=k)
        site = p.site()
        check("h", host(p.fwd()), site.h())
        check_grads(p, p.bwd(), site)
        if mode != "full":
            coef, dq = p.deferred()
            check("coef", host(coef), site.coef())
            check("dq", host(dq), site.dq())


def test_graph_replays(dev):
    """A decode step (append) and a backward in one captured graph, replayed with
    new inputs and eager work in between."""
    p = Problem(dev, "projected", "fp8", "bf16", 9, 6, 256, 16)
    S, N, d = p.cache.shape
    o = torch.zeros((N, d), dtype=torch.bfloat16, device=dev)
    H = torch.zeros_like(o)
    dV = torch.zeros((S, N, d), dtype=torch.bfloat16, device=dev)
    dK, dq = torch.zeros_like(p.K), torch.zeros_like(p.q)
    coef, dq2 = torch.zeros((S, 3, N), device=dev), torch.zeros_like(p.q)
    ws = torch.zeros((lr.cache_route_bwd_workspace_bytes(S, N, d, 16, "projected", "fp8",
                                                        torch.bfloat16),), dtype=torch.uint8, device=dev)

    def step():
        p.fwd(o_new=o, out=H)
        p.bwd(out=(dV, dK, dq), workspace=ws)
        lr.cache_route_bwd_deferred(p.cache, p.K, p.q, p.dH, p.mode, coef, dq=dq2, workspace=ws)

    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    outs = (H, dV, dK, dq, coef, dq2, p.cache.codes, p.cache.scales)
    rng = np.random.default_rng(1)
    for _ in range(4):
        o.copy_(torch.from_numpy(rng.standard_normal((N, d)).astype(np.float32)))
        p.dH.copy_(torch.from_numpy(rng.standard_normal((N, d)).astype(np.float32)))
        g.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in outs]
        for x in outs[:6]:
            x.fill_(float("nan"))
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, outs))


@pytest.mark.parametrize("fmt,mode", [("fp8", "projected"), ("fp4", "sliced"), ("fp8", "full")])
def test_beyond_two_to_the_31(dev, fmt, mode):
    """A stack of more than 2^31 values: sampled tokens, the last among them."""
    S, N, d, r = 41, 26000, 2056, 16
    assert S * N * d > 2 ** 31
    gen = torch.Generator(device=dev).manual_seed(4)
    cache = lr.source_cache(S, N, d, fmt, dev)
    cache.codes.random_(0, 256, generator=gen)
    if fmt == "fp8":
        cache.codes.bitwise_and_(0xF7)  # no NaN code
        cache.codes.clamp_(max=0xF6)
    cache.codes.view(S, N, -1)[..., -12 if fmt == "fp4" else -24:] = 0  # past the row
    cache.scales.random_(118, 122, generator=gen)
    r = d if mode == "full" else r
    q = torch.randn(r, generator=gen, device=dev) / r ** 0.5
    K = torch.randn(S, N, r, generator=gen, device=dev).bfloat16() if mode == "projected" else None
    dH = torch.randn(N, d, generator=gen, device=dev).bfloat16()
    print(f"case {mode} {fmt} beyond 2^31", flush=True)
    h = lr.cache_route_fwd(cache, K, q, mode)
    dV, dK, dq = lr.cache_route_bwd(cache, K, q, dH, mode)
    x = lr.cache_read(cache)
    torch.cuda.synchronize()
    pick = torch.tensor([0, 1, N // 2, N - 2, N - 1], device=dev)
    V = values(cache.codes[:, pick].cpu().numpy(), cache.scales[:, pick].cpu().numpy(), d, fmt)
    assert np.array_equal(host(x[:, pick]), V)
    site = Site(V, None if K is None else host(K[:, pick]), host(q), r, EPS, "bf16", host(dH[pick]))
    check("h", host(h[pick]), site.h())
    check("dV", host(dV[:, pick]), site.dV())
    if K is not None:
        check("dK", host(dK[:, pick]), site.dK())
    assert torch.isfinite(dq).all()


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("mode,dtype", [("projected", "bf16"), ("sliced", "f32")])
def test_model_pass(dev, mode, dtype, fmt):
    """A model pass as training runs it: every output joins the cache at the site
    that first reads it, then the deferred reverse pass with one gather a source,
    against the sum over sites of the 64-bit gradients."""
    T, N, d, r = 7, 37, 136, 24
    rng = np.random.default_rng(11)
    cache = lr.source_cache(T, N, d, fmt, dev)
    outs = [stored(rng.standard_normal((N, d)), dtype, dev) for _ in range(T)]
    K, k = stored(rng.standard_normal((T, N, r)), dtype, dev) if mode == "projected" else (None, None)
    Q = torch.from_numpy((rng.standard_normal((T, r)) / 5).astype(np.float32)).to(dev)
    dHs, dh = stored(rng.standard_normal((T, N, d)), dtype, dev)
    V = values(*quantise(np.stack([x for _, x in outs]), fmt), d, fmt)
    sub = lambda x, t: None if x is None else x[:t]  # noqa: E731
    sites = [Site(V[:t], sub(k, t), host(Q[t - 1]), r, EPS, dtype, dh[t - 1]) for t in range(1, T + 1)]
    for t in range(1, T + 1):
        h = lr.cache_route_fwd(cache.planes(0, t), sub(K, t), Q[t - 1], mode, o_new=outs[t - 1][0])
        check(f"h {t}", host(h), sites[t - 1].h())
    coefs = torch.zeros((T, T, 3, N), device=dev)
    for t in range(T, 0, -1):
        dq = lr.cache_route_bwd_deferred(cache.planes(0, t), sub(K, t), Q[t - 1], dHs[t - 1], mode,
                                         coefs[t - 1, :t])
        check(f"dq {t}", host(dq), sites[t - 1].dq())
        i = t - 1
        plane = lr.cache_read(cache.planes(i), DT[dtype])
        assert np.array_equal(host(plane[0]), V[i])
        dV, dK = lr.route_gather_bwd(plane, None if K is None else K[i:t], 0, dHs[i:], Q[i:],
                                     coefs[i:, i], mode)
        # The sum over the sites that read it, rounded once; its terms' bounds,
        # and n u of their sum for the gather's own additions.
        n = T - i
        want = [s.dV() for s in sites[i:]]
        x = sum(w[0][i] for w in want)
        half = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}[dtype]
        e = sum(w[1][i] - 2 * half * np.abs(w[0][i]) for w in want)  # without each site's rounding
        e = e + 2 * ((4 * n + 8) * 2.0 ** -24 * sum(np.abs(w[0][i]) for w in want)
                     + (4 * n + 8) * 2.0 ** -24 * _gather_terms(sites[i:], i, mode) + half * np.abs(x))
        check(f"dV {i}", host(dV), (x, e + 2.0 ** -120))
        if mode == "projected":
            want = [s.dK() for s in sites[i:]]
            x = sum(w[0][i] for w in want)
            e = sum(w[1][i] - 2 * half * np.abs(w[0][i]) for w in want)
            e = e + 2 * ((4 * n + 8) * 2.0 ** -24 * _key_terms(sites[i:], i) + half * np.abs(x))
            check(f"dK {i}", host(dK), (x, e + 2.0 ** -120))


def _key_terms(sites, i):
    return sum(np.abs(s.cq[i])[:, None] * np.abs(s.q) + np.abs(s.ck[i])[:, None] * np.abs(s.kbar[i])
               for s in sites)


def _gather_terms(sites, i, mode):
    x = sum(s.alpha[i][:, None] * np.abs(s.dH) for s in sites)
    if mode == "sliced":
        x[:, x.shape[1] - sites[0].r:] += _key_terms(sites, i)
    return x


@pytest.mark.parametrize("mode", ["projected", "sliced", "full"])
@pytest.mark.parametrize("S,N", [(5, 6), (35, 6), (5, 2100)])
def test_nan_and_huge_values_in_4_bits_stay_with_their_token(dev, mode, S, N):
    """As above over e2m1, whose full-rank dots of 16 sources share a product: a NaN
    block, then (full rank) a gradient above 1.5 * 2^127, which counts as infinite."""
    p = Problem(dev, mode, "fp4", "f32", S, N, 96, 16)
    clean, grads = p.fwd(), p.bwd()
    keep = torch.arange(N, device=dev) != 1
    p.cache.scales[2, 1, 2] = 255
    h, (dV, dK, dq) = p.fwd(), p.bwd()
    assert torch.equal(h[keep], clean[keep])
    assert torch.equal(dV[:, keep], grads[0][:, keep])
    assert h[1, 64:].isnan().all() and dq.isnan().any()
    if mode != "full":
        return
    assert h[1].isnan().all() and dV[:, 1].isnan().any()
    p = Problem(dev, mode, "fp4", "f32", S, N, 96, 16)
    p.dH[1, 40] = 3e38
    dV, _, dq = p.bwd()
    assert torch.equal(dV[:, keep], grads[0][:, keep])
    assert not dV[:, 1].isfinite().all() and not dq.isfinite().all()


@pytest.mark.parametrize("mode,d,r", [("sliced", 40, 9), ("projected", 700, 16), ("full", 100, 100),
                                      ("full", 700, 700)])
@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
@pytest.mark.parametrize("S", [1, 3, 4, 5, 8, 9, 12, 13, 16, 17, 20, 21, 41])
def test_forward_of_every_number_of_trips(dev, mode, d, r, fmt, S):
    """One wave a token, whose loads run ahead by a trip of four sources: no, one and
    two buffers in use, odd and even numbers of trips, a last one that is not full."""
    p = Problem(dev, mode, fmt, "bf16", S, 1030, d, r)
    check("h", host(p.fwd()), p.site(grad=False).h())

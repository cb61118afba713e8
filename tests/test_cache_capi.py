"""The source stack in 8 and 4 bits on the CPU: include/lr_attnres_cache.h is
exported, every invalid call is refused during host-side validation (no device
is touched), and the Python binding refuses wrong shapes, types and devices."""
import os
import re
import subprocess

import pytest

import paper_2607_09694_amd as lr

torch = pytest.importorskip("torch")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "lr_attnres_cache.h")
EINVAL, EUNSUPPORTED = 1, 2
P, SL, F = lr.PROJECTED, lr.SLICED, lr.FULL
BF16, F32 = 1, 0
FP8, FP4 = lr.FP8, lr.FP4

# Distinct fake device addresses; validation only compares them.
C, E, K, Q, G, H, DV, DK, DQ, WS, ON, CF = (0x10_0000_0000 * k for k in range(1, 13))


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(lr.LIB_PATH):
        from paper_2607_09694_amd.build import build

        build()
    return lr.load_library()


def err(lib):
    return lib.lr_attnres_last_error().decode()


def test_exports_every_declared_symbol(lib):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(lr_attnres_\w+)\s*\(", text)))
    assert names == ["lr_attnres_cache_read", "lr_attnres_cache_route_bwd",
                     "lr_attnres_cache_route_bwd_deferred",
                     "lr_attnres_cache_route_bwd_workspace_bytes", "lr_attnres_cache_route_fwd",
                     "lr_attnres_cache_row_bytes", "lr_attnres_cache_row_scales",
                     "lr_attnres_cache_write"]
    out = subprocess.run(["nm", "-D", "--defined-only", lr.LIB_PATH], capture_output=True,
                         text=True, check=True).stdout
    exported = set(re.findall(r"\sT\s+(\w+)", out))
    assert set(names) <= exported


def test_header_is_c(tmp_path):
    src = tmp_path / "a.c"
    src.write_text('#include "lr_attnres_cache.h"\nint main(void) { return LRAR_CACHE_FP4 - 1; }\n')
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"),
                    str(src), "-c", "-o", str(tmp_path / "a.o")], check=True)


def test_row_sizes(lib):
    for d in (1, 31, 32, 33, 1000, 1024, 2048):
        nb = -(-d // 32)
        assert lib.lr_attnres_cache_row_scales(d) == nb
        assert lib.lr_attnres_cache_row_bytes(d, FP8) == 32 * nb
        assert lib.lr_attnres_cache_row_bytes(d, FP4) == 16 * nb
    assert lib.lr_attnres_cache_row_bytes(0, FP8) == 0
    assert lib.lr_attnres_cache_row_bytes(64, 2) == 0
    assert lib.lr_attnres_cache_row_scales(-1) == 0


def copy(lib, write=True, O=G, codes=C, scales=E, rows=8, d=64, fmt=FP8, dtype=BF16):
    if write:
        return lib.lr_attnres_cache_write(O, codes, scales, rows, d, fmt, dtype, None)
    return lib.lr_attnres_cache_read(codes, scales, O, rows, d, fmt, dtype, None)


COPY_INVALID = [
    ("O NULL", dict(O=None), "O is NULL"),
    ("codes NULL", dict(codes=None), "codes is NULL"),
    ("scales NULL", dict(scales=None), "scales is NULL"),
    ("format", dict(fmt=2), "format"),
    ("storage", dict(dtype=3), "storage"),
    ("rows negative", dict(rows=-1), "sizes"),
    ("d zero", dict(d=0), "sizes"),
    ("codes misaligned", dict(codes=C + 8), "aligned"),
    ("O misaligned", dict(O=G + 1), "aligned"),
    ("O overlaps codes", dict(O=C + 64), "overlap"),
    ("O overlaps scales", dict(scales=G + 2), "overlap"),
    ("overflow", dict(rows=1 << 45, d=1 << 18), "overflow"),
    ("width overflow", dict(d=(1 << 63) - 1, rows=1), "overflow"),
]


@pytest.mark.parametrize("write", [True, False], ids=["write", "read"])
@pytest.mark.parametrize("name,kw,msg", COPY_INVALID, ids=[c[0] for c in COPY_INVALID])
def test_copy_rejects(lib, write, name, kw, msg):
    assert copy(lib, write, **kw) == EINVAL
    assert msg in err(lib)


@pytest.mark.parametrize("write", [True, False], ids=["write", "read"])
def test_copy_limits_and_empty(lib, write):
    far = dict(O=1 << 60, codes=1 << 58, scales=1 << 56)  # room for sizes like these
    assert copy(lib, write, rows=(1 << 40) + 1, d=32, **far) == EUNSUPPORTED
    assert copy(lib, write, rows=1, d=(1 << 20) + 1, **far) == EUNSUPPORTED
    assert copy(lib, write, rows=1 << 40, d=1 << 15, **far) == EUNSUPPORTED  # one launch
    assert copy(lib, write, rows=0, O=None, codes=None, scales=None) == 0


def test_write_overlapping_outputs(lib):
    assert copy(lib, scales=C + 16) == EINVAL
    assert "overlap" in err(lib)


def fwd(lib, codes=C, scales=E, K=None, q=Q, o_new=None, H=H, S=4, N=8, d=64, r=8, mode=SL, fmt=FP8,
        dtype=BF16, eps=1e-6):
    return lib.lr_attnres_cache_route_fwd(codes, scales, K, q, o_new, H, S, N, d, r, mode, fmt,
                                          dtype, eps, None)


def bwd(lib, codes=C, scales=E, K=None, q=Q, dH=G, dV=DV, dK=None, dq=DQ, ws=WS, wsb=1 << 30, S=4,
        N=8, d=64, r=8, mode=SL, fmt=FP8, dtype=BF16, eps=1e-6, acc=0):
    return lib.lr_attnres_cache_route_bwd(codes, scales, K, q, dH, dV, dK, dq, ws, wsb, S, N, d, r,
                                          mode, fmt, dtype, eps, acc, None)


def deferred(lib, codes=C, scales=E, K=None, q=Q, dH=G, coef=CF, dq=DQ, ws=WS, wsb=1 << 30, S=4, N=8,
             d=64, r=8, mode=SL, fmt=FP8, dtype=BF16, eps=1e-6):
    return lib.lr_attnres_cache_route_bwd_deferred(codes, scales, K, q, dH, coef, dq, ws, wsb, S, N,
                                                   d, r, mode, fmt, dtype, eps, None)


SITE_INVALID = [
    ("codes NULL", dict(codes=None), "codes is NULL"),
    ("scales NULL", dict(scales=None), "scales is NULL"),
    ("q NULL", dict(q=None), "q is NULL"),
    ("format", dict(fmt=-1), "format"),
    ("S zero", dict(S=0), "sizes"),
    ("N negative", dict(N=-1), "sizes"),
    ("sliced r > d", dict(r=65), "r <= d"),
    ("full r != d", dict(mode=F, r=8), "r == d"),
    ("K outside projected", dict(K=K), "K must be NULL"),
    ("projected without K", dict(mode=P), "K is NULL"),
    ("unknown mode", dict(mode=7), "mode"),
    ("unknown storage", dict(dtype=5), "storage"),
    ("eps nan", dict(eps=float("nan")), "eps"),
    ("eps negative", dict(eps=-1.0), "eps"),
    ("codes misaligned", dict(codes=C + 8), "aligned"),
    ("q misaligned", dict(q=Q + 2), "aligned"),
    ("overflow", dict(S=1 << 40, N=1 << 20, d=1 << 10), "overflow"),
]


@pytest.mark.parametrize("call", [fwd, bwd, deferred], ids=["fwd", "bwd", "deferred"])
@pytest.mark.parametrize("name,kw,msg", SITE_INVALID, ids=[c[0] for c in SITE_INVALID])
def test_site_rejects(lib, call, name, kw, msg):
    assert call(lib, **kw) == EINVAL
    assert msg in err(lib)


FWD_INVALID = [
    ("H NULL", dict(H=None), "H is NULL"),
    ("H misaligned", dict(H=H + 8), "aligned"),
    ("o_new misaligned", dict(o_new=ON + 2), "aligned"),
    ("H overlaps codes", dict(H=C + 16), "overlap"),
    ("H overlaps o_new", dict(o_new=H + 16), "overlap"),
    ("o_new overlaps the cache", dict(o_new=C + 32), "overlap"),
    ("codes overlap scales", dict(scales=C + 1), "overlap"),
    ("q inside the cache", dict(q=C + 32), "overlap"),
]


@pytest.mark.parametrize("name,kw,msg", FWD_INVALID, ids=[c[0] for c in FWD_INVALID])
def test_forward_rejects(lib, name, kw, msg):
    assert fwd(lib, **kw) == EINVAL
    assert msg in err(lib)


BWD_INVALID = [
    ("dH NULL", dict(dH=None), "dH is NULL"),
    ("dq NULL", dict(dq=None), "dq is NULL"),
    ("dH misaligned", dict(dH=G + 2), "aligned"),
    ("workspace too small", dict(wsb=4), "workspace"),
    ("workspace NULL", dict(ws=None), "workspace"),
    ("workspace misaligned", dict(ws=WS + 4), "aligned"),
    ("workspace overlaps codes", dict(ws=C + 64), "overlap"),
    ("dq overlaps q", dict(dq=Q), "overlap"),
]
GRAD_INVALID = [
    ("dV NULL", dict(dV=None), "dV is NULL"),
    ("dV misaligned", dict(dV=DV + 4), "aligned"),
    ("dV overlaps codes", dict(dV=C), "overlap"),
    ("dV overlaps dH", dict(dV=G), "overlap"),
    ("dq inside dV", dict(dq=DV + 16), "overlap"),
    ("dK outside projected", dict(dK=DK), "must be NULL"),
    ("projected without dK", dict(mode=P, K=K), "dK is NULL"),
    ("accumulate", dict(acc=2), "accumulate"),
]
COEF_INVALID = [
    ("coef NULL", dict(coef=None), "coef is NULL"),
    ("coef misaligned", dict(coef=CF + 2), "aligned"),
    ("coef overlaps scales", dict(coef=E + 4), "overlap"),
    ("dq inside coef", dict(dq=CF + 8), "overlap"),
]


@pytest.mark.parametrize("call,name,kw,msg",
                         [(bwd, *c) for c in BWD_INVALID + GRAD_INVALID]
                         + [(deferred, *c) for c in BWD_INVALID + COEF_INVALID],
                         ids=[f"bwd {c[0]}" for c in BWD_INVALID + GRAD_INVALID]
                         + [f"deferred {c[0]}" for c in BWD_INVALID + COEF_INVALID])
def test_backward_rejects(lib, call, name, kw, msg):
    assert call(lib, **kw) == EINVAL
    assert msg in err(lib)


def test_unsupported(lib):
    assert fwd(lib, S=1025) == EUNSUPPORTED
    assert fwd(lib, N=(1 << 25) + 1, S=1, d=8, r=8) == EUNSUPPORTED
    assert fwd(lib, d=(1 << 20) + 1) == EUNSUPPORTED
    assert fwd(lib, mode=F, d=4097, r=4097) == EUNSUPPORTED
    for call in (bwd, deferred):
        assert call(lib, S=513) == EUNSUPPORTED
        assert call(lib, r=257, d=1024) == EUNSUPPORTED
        assert call(lib, d=4097) == EUNSUPPORTED
    assert bwd(lib, mode=F, d=4097, r=4097) == EUNSUPPORTED
    assert deferred(lib, mode=F, r=64) == EUNSUPPORTED
    assert "deferred" in err(lib)


def test_workspace_query(lib):
    q = lib.lr_attnres_cache_route_bwd_workspace_bytes
    for mode, r in ((P, 32), (SL, 32), (F, 512)):
        for N in (1, 511, 512, 513, 4095, 4096, 16384):
            sizes = [q(S, N, 512, r, mode, FP8, BF16) for S in (1, 8, 9, 64, 129, 512)]
            assert sizes == sorted(sizes) and sizes[0] > 0
    assert q(4, 0, 64, 8, SL, FP8, BF16) == 0
    assert q(4, 8, 64, 8, 9, FP8, BF16) == 0
    assert q(4, 8, 64, 8, SL, 7, BF16) == 0
    assert q(513, 8, 64, 8, SL, FP8, BF16) == 0


# The binding, on CPU tensors: what it refuses before the library is called.

def make(S=3, N=5, d=40, fmt="fp8"):
    return lr.source_cache(S, N, d, fmt, device="cpu")


def test_source_cache_shapes():
    c = make(fmt="fp4")
    assert c.shape == (3, 5, 40) and c.codes.shape == (3, 5, 32) and c.scales.shape == (3, 5, 2)
    assert c.planes(-1).codes.data_ptr() == c.codes[2].data_ptr()
    assert c.planes(0, 2).shape == (2, 5, 40)
    assert c.planes(3, 0).shape == (0, 5, 40)
    for bad in ((3, 1), (-4, 1), (1, 3), (0, -1)):
        with pytest.raises(ValueError):
            c.planes(*bad)
    with pytest.raises(ValueError):
        lr.SourceCache(c.codes, c.scales, 65, "fp4")
    with pytest.raises(ValueError):
        lr.SourceCache(c.codes, c.scales, 40, "fp8")
    with pytest.raises(ValueError):
        lr.SourceCache(c.codes, c.scales[:2], 40, "fp4")
    with pytest.raises(TypeError):
        lr.SourceCache(c.codes.int(), c.scales, 40, "fp4")
    with pytest.raises((ValueError, KeyError)):
        lr.SourceCache(c.codes, c.scales, 40, "int8")


def test_binding_refuses(lib):
    c, q = make(), torch.zeros(8)
    O, dH = torch.zeros(3, 5, 40).bfloat16(), torch.zeros(5, 40).bfloat16()
    Kt = torch.zeros(3, 5, 8).bfloat16()
    with pytest.raises(ValueError, match="device"):
        lr.cache_write(c, O)
    with pytest.raises(ValueError, match="O must be"):
        lr.cache_write(c, O[:2])
    with pytest.raises(ValueError, match="out must be"):
        lr.cache_read(c, out=O[..., :39])
    with pytest.raises(TypeError):
        lr.cache_read(c, dtype=torch.float32, out=O)
    with pytest.raises(ValueError, match="K must be"):
        lr.cache_route_fwd(c, None, q, "projected")
    with pytest.raises(ValueError, match="K must be None"):
        lr.cache_route_fwd(c, Kt, q, "sliced")
    with pytest.raises(ValueError, match="K must be"):
        lr.cache_route_fwd(c, Kt[:2], q, "projected")
    with pytest.raises(ValueError, match="q must"):
        lr.cache_route_fwd(c, Kt, q[:7], "projected")
    with pytest.raises(ValueError, match="o_new must be"):
        lr.cache_route_fwd(c, None, q, "sliced", o_new=dH[:4])
    with pytest.raises(ValueError, match="out must be"):
        lr.cache_route_fwd(c, None, q, "sliced", out=dH[:4])
    with pytest.raises(ValueError, match="dH must be"):
        lr.cache_route_bwd(c, None, q, dH[:4], "sliced")
    with pytest.raises(ValueError, match="accumulate"):
        lr.cache_route_bwd(c, None, q, dH, "sliced", accumulate=True)
    with pytest.raises(ValueError, match="dK"):
        lr.cache_route_bwd(c, Kt, q, dH, "projected", out=(O, None, q))
    with pytest.raises(ValueError, match="dV must be"):
        lr.cache_route_bwd(c, None, q, dH, "sliced", out=(O[:2], None, q))
    with pytest.raises(ValueError, match="dq must be"):
        lr.cache_route_bwd(c, None, q, dH, "sliced", out=(O, None, q[:3]))
    with pytest.raises(ValueError, match="coef must be"):
        lr.cache_route_bwd_deferred(c, None, q, dH, "sliced", torch.zeros(3, 5, 3))

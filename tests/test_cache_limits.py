"""What the calls over the 8- and 4-bit stack refuse before a device is touched: formats
and storages that do not exist, by one kind of error each, and the documented limits."""
import pytest

import paper_2607_09694_amd as lr
from test_cache_capi import EUNSUPPORTED, FP4, FP8, K, P, err, fwd, lib, make  # noqa: F401

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("fmt", ["int8", "FP8", "", 2, -1])
def test_unknown_formats(lib, fmt):  # noqa: F811
    c = make()
    for call in (lambda: lr.SourceCache(c.codes, c.scales, 40, fmt),
                 lambda: lr.source_cache(3, 5, 40, fmt, device="cpu"),
                 lambda: lr.cache_route_bwd_workspace_bytes(4, 8, 64, 8, "sliced", fmt, torch.bfloat16)):
        with pytest.raises(ValueError, match="cache format"):
            call()


@pytest.mark.parametrize("dtype", [torch.float16, torch.float64, torch.uint8])
def test_workspace_query_refuses_other_storages(lib, dtype):  # noqa: F811
    with pytest.raises(TypeError, match="bfloat16 or float32"):
        lr.cache_route_bwd_workspace_bytes(4, 8, 64, 8, "sliced", "fp8", dtype)


def test_known_formats_by_name_and_number(lib):  # noqa: F811
    for name, number in (("fp8", FP8), ("fp4", FP4)):
        a, b = lr.source_cache(2, 3, 33, name, device="cpu"), lr.source_cache(2, 3, 33, number, device="cpu")
        assert a.fmt == b.fmt == number and a.codes.shape == b.codes.shape
        for dtype in (torch.bfloat16, torch.float32):
            need = lr.cache_route_bwd_workspace_bytes(4, 2000, 64, 8, "sliced", name, dtype)
            assert need == lr.cache_route_bwd_workspace_bytes(4, 2000, 64, 8, "sliced", number, dtype) > 0


def test_query_of_no_dimension(lib):  # noqa: F811
    c = make()
    with pytest.raises(ValueError, match="q must"):
        lr.cache_route_fwd(c, None, torch.zeros(()), "sliced")


def test_projected_key_width(lib):  # noqa: F811
    far = dict(codes=1 << 58, scales=1 << 56, H=1 << 50, o_new=None)  # room for the keys
    assert fwd(lib, mode=P, K=K, r=(1 << 20) + 1, S=2, N=1, q=1 << 55, **far) == EUNSUPPORTED
    assert "key width" in err(lib)


def test_row_sizes_of_rows_too_wide(lib):  # noqa: F811
    assert lib.lr_attnres_cache_row_scales(1 << 20) == 1 << 15
    assert lib.lr_attnres_cache_row_scales((1 << 20) + 1) == 0
    assert lib.lr_attnres_cache_row_bytes((1 << 20) + 1, FP8) == 0
    assert lib.lr_attnres_cache_row_bytes((1 << 20) + 1, FP4) == 0

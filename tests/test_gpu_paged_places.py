"""Pools without a place for every row: strides of 0 alone mean dense ones to the C calls, which would
read and write behind the one row that there is."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32, torch.float8_e4m3fn])
def test_expanded_pools_are_refused(lib, dtype):
    table = torch.zeros(2, 3, dtype=torch.int32, device=DEV)
    kw = {}
    if dtype is torch.float8_e4m3fn:
        scales = torch.full((2, 6, 2, 16), 127, dtype=torch.uint8, device=DEV).view(torch.float8_e8m0fnu)
        kw = dict(k_scales=scales[0], v_scales=scales[1])
    rows = torch.zeros(2, 6 * 2 * 16 * 64, dtype=torch.uint8, device=DEV).repeat(1, dtype.itemsize).view(dtype)
    full = rows.view(2, 6, 2, 16, 64)
    lib.PagedCache(full[0], full[1], table, **kw)
    one = full[:, :1, :1, :1].expand(2, 6, 2, 16, 64)
    assert one.stride()[1:4] == (0, 0, 0)
    with pytest.raises(ValueError):
        lib.PagedCache(one[0], one[1], table, **kw)
    if not kw:  # one row is one place
        lib.PagedCache(full[0, :1, :1, :1], full[1, :1, :1, :1], table)

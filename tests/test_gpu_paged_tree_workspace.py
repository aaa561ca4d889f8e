"""The workspace of ripple_paged_tree_attn grows with the call on this device."""
import ctypes

import pytest

pytestmark = pytest.mark.gpu


def _tree_bytes(lib, dtype, codes, hq, most, **over):
    a = dict(batch=1, n_kv_heads=1, head_dim=128, page_size=16, n_pages=40, max_pages=8, dtype=dtype,
             page_stride=0, head_stride=0, row_stride=0)
    a.update(over)
    n, s = ctypes.c_size_t(), lib.PagedScales(1 << 32, 1 << 33, 0, 0, 0)
    assert lib._lib.ripple_paged_tree_workspace_bytes(
        ctypes.byref(lib.PagedDesc(**a)), ctypes.byref(s) if codes else None, hq, most,
        ctypes.byref(n)) == lib.OK
    return n.value


@pytest.mark.parametrize("codes", [False, True])
def test_tree_workspace_serves_every_smaller_call(lib, codes):
    # on this device: tokens, heads, batches and tables that leave SMs over at some numbers of tiles
    for dtype in (lib.BF16, lib.F32):
        for G in (1, 7, 8, 16):
            for blocks in (1, 19, 40, 76, 152, 200, 303, 304, 400):
                sizes = [_tree_bytes(lib, dtype, codes, G, most, max_pages=4 * blocks)
                         for most in range(1, 65)]
                assert sizes == sorted(sizes), (G, blocks)
        for most in (1, 5, 33, 64):
            sizes = [_tree_bytes(lib, dtype, codes, G, most, max_pages=640) for G in range(1, 17)]
            assert sizes == sorted(sizes)
            sizes = [_tree_bytes(lib, dtype, codes, 8, most, max_pages=4 * b) for b in range(1, 500)]
            assert sizes == sorted(sizes)
            sizes = [_tree_bytes(lib, dtype, codes, 8, most, batch=b) for b in range(1, 400)]
            assert sizes == sorted(sizes)

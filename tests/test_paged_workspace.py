"""What the header says of the paged decode's workspace and of the sizes a cache may have."""
import ctypes

from tests.test_paged_host import _desc


def _need(lib, hkv, group, **over):
    n = ctypes.c_size_t()
    st = lib._lib.ripple_paged_decode_workspace_bytes(
        ctypes.byref(_desc(lib, n_kv_heads=hkv, **over)), hkv * group, ctypes.byref(n))
    return n.value if st == lib.OK else st


def test_the_largest_of_each_serves_all(lib):
    for d, dtype in ((64, lib.F32), (128, lib.BF16)):
        most = _need(lib, 33, 16, batch=70, max_pages=900, head_dim=d, dtype=dtype)
        for hkv in (1, 2, 3, 8, 32, 33):
            for group in (1, 2, 5, 8, 16):
                for batch in (1, 2, 9, 64, 70):
                    for pages in (1, 7, 64, 900):
                        assert _need(lib, hkv, group, batch=batch, max_pages=pages, head_dim=d,
                                     dtype=dtype) <= most
        for grow in ([_need(lib, h, 4, batch=9, head_dim=d, dtype=dtype) for h in range(1, 80)],
                     [_need(lib, 3, g, batch=9, head_dim=d, dtype=dtype) for g in range(1, 17)]):
            assert grow == sorted(grow)


def test_query_heads_alone_do_not_tell_it(lib):
    # once the runs are as many as they get, the same query heads on more KV heads need fewer
    # bytes: the header promises no order between these
    sizes = [_need(lib, h, 16 // h, batch=1000, max_pages=900) for h in (1, 2, 4, 8, 16)]
    assert sizes[-1] < sizes[0]


def test_groups_of_a_call(lib):
    assert _need(lib, 256, 1, batch=1 << 16) > 100
    assert _need(lib, 257, 1, batch=1 << 16) == lib.EINVAL  # batch * n_kv_heads above 2^24

"""Layers whose rows would be moved over one another's are refused when their tables are built; ones that
interleave in one buffer are not, and keep their rows apart."""
import pytest
import torch

from tests import paged8_common as P8
from tests import paged_common as P

pytestmark = pytest.mark.gpu
DEV = "cuda"
F8, E8 = torch.float8_e4m3fn, torch.float8_e8m0fnu


def _cache(lib, k, v, ks, vs, table):
    return lib.PagedCache(k.view(F8), v.view(F8), table, k_scales=ks.view(E8), v_scales=vs.view(E8))


def test_layers_that_share_scales_or_rows_are_refused(lib):
    a, b = (P8.Pool8(lib, [20, 20], 2, 64, 8, "bf16", 10 + i) for i in range(2))
    t = a.table
    lib.KeepTables([a.cache, b.cache])
    for ks, vs in ((a.ks, b.vs), (b.ks, a.vs), (a.vs, b.vs), (b.ks, a.ks), (b.ks, b.ks)):
        with pytest.raises(ValueError):
            lib.KeepTables([a.cache, _cache(lib, b.k, b.v, ks, vs, t)])
    # pools and scales that overlap in part, by a page or a row
    n = a.n_pages
    big = torch.zeros(2 * n, 2, 8, 64, dtype=torch.uint8, device=DEV)
    scales = torch.full((2 * n, 2, 8), 127, dtype=torch.uint8, device=DEV)
    for at in (1, n - 1):
        with pytest.raises(ValueError):
            lib.KeepTables([_cache(lib, big[:n], a.v, a.ks, a.vs, t),
                            _cache(lib, big[at:at + n], b.v, b.ks, b.vs, t)])
        with pytest.raises(ValueError):
            lib.KeepTables([_cache(lib, a.k, a.v, scales[:n], a.vs, t),
                            _cache(lib, b.k, b.v, b.ks, scales[at:at + n], t)])
    lib.KeepTables([_cache(lib, big[:n], a.v, scales[:n], a.vs, t),
                    _cache(lib, big[n:], b.v, scales[n:], b.vs, t)])
    x, y = (torch.zeros(2 * n, 2, 8, 64, dtype=torch.bfloat16, device=DEV) for _ in "kv")
    with pytest.raises(ValueError):
        lib.KeepTables([lib.PagedCache(x[:n], y[:n], t), lib.PagedCache(x[n - 1:-1], y[n:], t)])
    with pytest.raises(ValueError):  # one layer's values over the other's keys
        lib.KeepTables([lib.PagedCache(x[:n], y[:n], t), lib.PagedCache(y[n // 2:n // 2 + n], x[n:], t)])


@pytest.mark.parametrize("codes", [False, True])
def test_layers_side_by_side_in_one_buffer(lib, codes):
    # [pages][layers][K, V][heads][rows][d], the scales alike
    L, n_pages, H, page, d, B, n = 3, 12, 2, 16, 64, 2, 5
    kind = torch.uint8 if codes else torch.bfloat16
    pool = torch.randint(0, 120, (n_pages, L, 2, H, page, d), dtype=torch.uint8, device=DEV).to(kind)
    scales = torch.randint(100, 130, (n_pages, L, 2, H, page), dtype=torch.uint8, device=DEV)
    tables = [torch.randperm(n_pages, device=DEV)[:B * 4].int().view(B, 4) for _ in range(L)]
    caches = [_cache(lib, pool[:, l, 0], pool[:, l, 1], scales[:, l, 0], scales[:, l, 1], tables[l])
              if codes else lib.PagedCache(pool[:, l, 0], pool[:, l, 1], tables[l]) for l in range(L)]
    lens = [[40, 64], [20, 33], [5, 50]]
    want, want_s = pool.clone(), scales.clone()
    path = [[0, 2, 4], [3, 4]]
    for l in range(L):
        for b in range(B):
            first = lens[l][b] - n
            for j, x in enumerate(path[b]):
                src, dst = first + x, first + j
                (sp, ss), (dp, ds) = ((int(tables[l][b, r // page]), r % page) for r in (src, dst))
                want[dp, l, :, :, ds] = want[sp, l, :, :, ss].clone()
                want_s[dp, l, :, :, ds] = want_s[sp, l, :, :, ss].clone()
    lens_t, st = P.i32(lens), torch.zeros(1, dtype=torch.int32, device=DEV)
    lib.ripple_paged_keep_rows(lib.KeepTables(caches), lens_t, P.i32([[0, 2, 4], [3, 4, -1]]), n_tokens=n,
                               dev_status=st)
    assert int(st.item()) == 0 and torch.equal(pool, want)
    assert torch.equal(scales, want_s if codes else scales)
    assert lens_t.tolist() == [[a - n + 3, b - n + 2] for a, b in lens]

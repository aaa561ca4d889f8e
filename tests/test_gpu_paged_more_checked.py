"""The 8-bit pages', the drafts' and the kept rows' kernels in the bounds-checked build: no access
out of range, and the normal build's outputs bit for bit; and their waits giving up."""
import numpy as np
import pytest
import torch

from tests import paged8_common as P8
from tests import paged_common as P
from tests.test_gpu_checked import chk  # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("kind,G,H,d,page,lens", [
    ("q8-bf16", 4, 2, 128, 16, [0, 3, 700, 33, 4000, 15]), ("q8-bf16", 7, 3, 64, 8, [5000, 2, 100]),
    ("q8-f32", 16, 1, 128, 64, [9001]), ("q8-f32", 2, 2, 64, 1, [40, 3000]),
    ("bf16", 8, 2, 128, 32, [333, 0, 1200]), ("bf16", 5, 2, 64, 4, [64, 65, 9]),
    ("f32", 4, 2, 64, 16, [40, 3000]), ("f32", 16, 1, 128, 1024, [700])])
def test_calls_checked(lib, chk, kind, G, H, d, page, lens):
    B, n, t = len(lens), 2, P8.type_of(kind)
    q = P.randn((B, n, G * H, d), t, 70)
    kn, vn = P.randn((B, n, H, d), t, 71), P.randn((B, n, H, d), t, 72)
    inv = [10000.0 ** (-2.0 * j / d) for j in range(d // 2)]
    runs = []
    for m in (lib, chk):
        pool = P8.any_pool(m, kind, lens, H, d, page, 73)
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        q_out = torch.empty_like(q)
        lens_t = P.i32([lens])
        m.ripple_paged_append(pool.cache, lens_t[0], kn, vn, rope=m.Rope(inv), q=q, q_out=q_out,
                              dev_status=status)
        masks = P8.to_i64([1, 2] * B).view(B, n)
        tree, tree_lse, _ = P8.run_tree(m, pool, q_out, lens_t[0], masks, status=status)
        out, lse, _ = P.run_decode(m, pool, q_out[:, 0], lens_t[0], status=status)
        m.ripple_paged_keep_rows(m.KeepTables([pool.cache]), lens_t, P.i32([[1]] * B), n_tokens=n,
                                 dev_status=status)
        torch.cuda.synchronize()
        held = [getattr(pool, x) for x in ("k", "v", "ks", "vs") if hasattr(pool, x)]
        runs.append((int(status.item()), q_out, tree, tree_lse, out, lse, lens_t, *held))
    assert runs[1][0] == 0
    assert all(torch.equal(x, y) for x, y in zip(runs[0][1:], runs[1][1:]))


@pytest.mark.parametrize("kind", ["bf16", "q8-bf16"])
def test_waits_give_up(lib, kind):
    # waits of the tensor-core kernel out of time: reported, and the next call is as ever. (A
    # poll may suspend a thread for longer than a short bound, so the GPU is kept busy: a block
    # takes its CTA microseconds.)
    lens, counts = [40000] * 6 + [500], [30] * 7
    pool = P8.any_pool(lib, kind, [3000] * 6 + [500], 8, 128, 64, 80)
    pool.table = torch.from_numpy(np.concatenate([pool.np_table] * 15, 1)).to(DEV)  # pages again and again
    pool.table[6, 8:] = -1
    if kind == "bf16":
        pool.cache = lib.PagedCache(pool.k, pool.v, pool.table)
    else:
        pool.bind()
    q = P.randn((210, 32, 128), "bf16", 81)
    starts = P.i32([0] + np.cumsum(counts).tolist())
    want, want_lse, st = P8.run_tree(lib, pool, q, P.i32(lens), None, starts, 30)
    assert int(st.item()) == 0
    for limit in (100, 400):
        before = lib.ripple_set_wait_limit_cycles(limit)
        try:
            _, _, st = P8.run_tree(lib, pool, q, P.i32(lens), None, starts, 30)
            torch.cuda.synchronize()
        finally:
            lib.ripple_set_wait_limit_cycles(before)
        assert int(st.item()) == lib.ETIMEOUT, limit
        out, lse, st = P8.run_tree(lib, pool, q, P.i32(lens), None, starts, 30)
        assert int(st.item()) == 0
        assert torch.equal(out, want) and torch.equal(lse, want_lse)

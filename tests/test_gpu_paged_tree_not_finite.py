"""One value in a long cache that is not finite: the outputs are what the sum is, and the call takes about
as long as looking at its values again takes."""
import time

import numpy as np
import pytest
import torch

from tests import paged8_common as P8
from tests import paged_common as P

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _seconds(f):
    f()
    best = 1e9
    for _ in range(3):
        torch.cuda.synchronize()
        t = time.perf_counter()
        f()
        torch.cuda.synchronize()
        best = min(best, time.perf_counter() - t)
    return best


@pytest.mark.parametrize("n,d", [(8, 128), (16, 128), (16, 64), (32, 128)])
def test_one_value_in_long_caches(lib, n, d):
    # 64 sequences of 20000 rows, the same pages again and again, so that a part is thousands of rows
    B, H, G, page, rows = 64, 8, 4, 64, 20000
    pool = P.Pool(lib, [2048], H, d, page, "bf16", 11, "heads")
    width = -(-rows // page)
    entries = np.resize(pool.np_table[0, :32], width).astype(np.int32)
    table = torch.from_numpy(entries).to(DEV).expand(B, width).contiguous()
    cache = lib.PagedCache(pool.k, pool.v, table)
    q = P.randn((B, n, H * G, d), "bf16", 12)
    lens = P.i32([rows - 300 * b for b in range(B)])
    ws = torch.empty(lib.ripple_paged_tree_workspace_bytes(cache, H * G, n), dtype=torch.uint8, device=DEV)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    out = torch.empty_like(q)
    call = lambda: lib.ripple_paged_tree_attn(cache, q, lens, out, ws, dev_status=st)  # noqa: E731
    plain = _seconds(call)
    base = out.clone()
    inf, nan = float("inf"), float("nan")
    p = int(pool.np_table[0, 3])
    for head, dims in ((2, {5: inf}), (6, {0: -inf, 33: nan, 63: inf})):
        for at, x in dims.items():
            pool.v[p, head, 17, at] = x
    took = _seconds(call)
    assert int(st.item()) == 0
    for head in range(H):
        mine = out[:, :, head * G:(head + 1) * G]
        want = base[:, :, head * G:(head + 1) * G].clone()
        for at, x in {2: {5: inf}, 6: {0: -inf, 33: nan, 63: inf}}.get(head, {}).items():
            want[..., at] = x
        assert torch.equal(torch.nan_to_num(mine.float(), 7e30, 8e30, 9e30),
                           torch.nan_to_num(want.float(), 7e30, 8e30, 9e30)), head
    assert took < 25 * plain, (took, plain)

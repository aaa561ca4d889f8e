"""Waits of the trees' tensor-core kernel out of time: every call comes back, with what its CTAs still had
on its way landed, and the next call is as ever. Query rows in four copies, in two and in one;
long caches by runs, short ones by clusters, whose few blocks are all fetched before any wait for
room (a role then gives up on loads whose own warp is done).

A poll may suspend a thread for longer than a short bound, so that whether a short call's waits
run out depends on the run; a long one's do."""
import time

import numpy as np
import pytest
import torch

from tests import paged8_common as P8
from tests import paged_common as P

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _call(lib, pool, q, lens, starts, most, limit):
    """The call with a bound for its waits: status, seconds until it is back."""
    before = lib.ripple_set_wait_limit_cycles(limit)
    try:
        t = time.perf_counter()
        _, _, st = P8.run_tree(lib, pool, q, P.i32(lens), None, starts, most)
        torch.cuda.synchronize()
        t = time.perf_counter() - t
    finally:
        lib.ripple_set_wait_limit_cycles(before)
    return int(st.item()), t


@pytest.mark.parametrize("kind", ["bf16", "q8-bf16"])
@pytest.mark.parametrize("n", [8, 16, 32])
@pytest.mark.parametrize("short", [False, True])
def test_calls_out_of_time_come_back(lib, short, n, kind):
    if short:
        rows, lens, repeat = [100, 128, 70, 64], [100, 128, 70, 64], 1
    else:
        rows, lens, repeat = [3000] * 6 + [500], [40000] * 6 + [500], 15
    pool = P8.any_pool(lib, kind, rows, 8, 128, 64, 80)
    if repeat > 1:  # pages again and again
        pool.table = torch.from_numpy(np.concatenate([pool.np_table] * repeat, 1)).to(DEV)
        pool.table[6, 8:] = -1
        if kind == "bf16":
            pool.cache = lib.PagedCache(pool.k, pool.v, pool.table)
        else:
            pool.bind()
    counts = [n - i % 3 for i in range(len(lens))]
    q = P.randn((sum(counts), 32, 128), "bf16", 81)
    starts = P.i32([0] + np.cumsum(counts).tolist())
    want, want_lse, st = P8.run_tree(lib, pool, q, P.i32(lens), None, starts, n)
    assert int(st.item()) == 0
    seen = set()
    for limit in (1, 100, 400, 1000, 3000):
        for _ in range(3):
            status, seconds = _call(lib, pool, q, lens, starts, n, limit)
            assert status in (0, lib.ETIMEOUT) and seconds < 5, limit
            seen.add(status)
        out, lse, st = P8.run_tree(lib, pool, q, P.i32(lens), None, starts, n)
        assert int(st.item()) == 0
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
    assert short or lib.ETIMEOUT in seen

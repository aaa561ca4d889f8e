"""The paged operators and the log probabilities in the bounds-checked build: no access out
of range, and the normal build's outputs bit for bit."""
import pytest
import torch

from tests import paged_common as P
from tests.test_gpu_checked import chk  # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("dtype,G,H,d,page,lens", [
    ("bf16", 4, 2, 128, 16, [0, 1, 700, 33, 4000, 15]), ("bf16", 7, 3, 64, 8, [5000, 2, 100]),
    ("bf16", 16, 1, 128, 64, [9001]), ("f32", 8, 2, 128, 32, [333, 0, 1200]),
    ("f32", 1, 2, 64, 1, [40, 3000])])
def test_paged_calls_checked(lib, chk, dtype, G, H, d, page, lens):
    B = len(lens)
    q = P.randn((B, 1, G * H, d), dtype, 70)
    kn, vn = P.randn((B, 1, H, d), dtype, 71), P.randn((B, 1, H, d), dtype, 72)
    inv = [10000.0 ** (-2.0 * j / d) for j in range(d // 2)]
    runs = []
    for m in (lib, chk):
        pool = P.Pool(m, lens, H, d, page, dtype, 73)
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        q_out = torch.empty_like(q)
        m.ripple_paged_append(pool.cache, P.i32(lens), kn, vn, rope=m.Rope(inv), q=q, q_out=q_out,
                              dev_status=status)
        out, lse, _ = P.run_decode(m, pool, q_out[:, 0], P.i32(lens), status=status)
        torch.cuda.synchronize()
        runs.append((int(status.item()), q_out, pool.k, pool.v, out, lse))
    assert runs[1][0] == 0
    assert all(torch.equal(x, y) for x, y in zip(runs[0][1:], runs[1][1:]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,V,stride", [(1, 128256, 128256), (9, 5003, 5007), (200, 1001, 1001), (3, 7, 7),
                                        (700, 2000, 2003)])
def test_logprobs_checked(lib, chk, n, V, stride, dtype):
    x = P.randn((n, stride), dtype, 80)[:, :V]
    tokens = P.i32([i % V for i in range(n)])
    runs = []
    for m in (lib, chk):
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        out = [torch.zeros(n, device=DEV) for _ in range(3)]
        idx = torch.zeros(n, 5, dtype=torch.int32, device=DEV)
        top = torch.zeros(n, 5, device=DEV)
        m.ripple_token_logprobs(x, tokens, out[0], out[1], out[2], idx, top, dev_status=status)
        torch.cuda.synchronize()
        runs.append((int(status.item()), *out, idx, top))
    assert runs[1][0] == 0
    assert all(torch.equal(x, y) for x, y in zip(runs[0][1:], runs[1][1:]))

"""The largest logit scale gives what it means."""
import math

import numpy as np
import pytest
import torch

from tests import paged_common as P

pytestmark = pytest.mark.gpu
DEV = "cuda"
BIG = 2.0 ** 127


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_log_probabilities(lib, dtype):
    # scaled logits 0, -2, -6 and one of which nothing is left
    x = torch.tensor([[0.0, -2.0 ** -126, -3 * 2.0 ** -126, -1.0]], device=DEV).to(P.DT[dtype])
    lp, ent, lse = (torch.zeros(1, device=DEV) for _ in range(3))
    idx, top = torch.zeros(1, 4, dtype=torch.int32, device=DEV), torch.zeros(1, 4, device=DEV)
    lib.ripple_token_logprobs(x, P.i32([1]), lp, ent, lse, idx, top, scale=BIG)
    torch.cuda.synchronize()
    s = math.log(1 + math.exp(-2) + math.exp(-6))
    assert idx[0].tolist() == [0, 1, 2, 3]
    # the kernel's own 2^-20 (test_gpu_logprobs.py); the entropy's terms, exp(-2) 2^-126 and
    # 3 exp(-6) 2^-126, are rounded to multiples of 2^-149: 2^-17 of the second at most
    np.testing.assert_allclose(top[0, :3].tolist(), [-s, -2 - s, -6 - s], rtol=2.0 ** -19)
    assert top[0, 3].item() == -BIG
    np.testing.assert_allclose([lp.item(), lse.item()], [-2 - s, s], rtol=2.0 ** -19)
    want = s + (2 * math.exp(-2) + 6 * math.exp(-6)) / math.exp(s)
    np.testing.assert_allclose(ent.item(), want, rtol=2.0 ** -17)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_decode(lib, dtype):
    # queries of 2^-63 against keys of 2^-63, 0 and -2^-63: scores 2, 0 and -2
    pool = P.Pool(lib, [3], 1, 64, 16, dtype, 5)
    page = int(pool.np_table[0, 0])
    pool.k.zero_()
    pool.k[page, 0, 0, 0], pool.k[page, 0, 2, 0] = 2.0 ** -63, -2.0 ** -63
    q = torch.zeros(1, 4, 64, device=DEV).to(P.DT[dtype])
    q[:, :, 0] = 2.0 ** -63
    out, lse, st = P.run_decode(lib, pool, q, P.i32([3]), scale=BIG)
    assert int(st.item()) == 0
    w = np.exp([2.0, 0.0, -2.0])
    want = (w[:, None] * pool.seq("v", 0)[0]).sum(0) / w.sum()
    np.testing.assert_allclose(out[0].cpu().numpy(), np.broadcast_to(want, (4, 64)), atol=1e-5)
    np.testing.assert_allclose(lse[0].cpu().numpy(), math.log(w.sum()), rtol=1e-5)


def test_scales_that_fp32_rounds_to_0_are_refused(lib):
    pool = P.Pool(lib, [3], 1, 64, 16, "f32", 5)
    q = torch.ones(1, 4, 64, device=DEV)
    with pytest.raises(ValueError, match="scale"):
        P.run_decode(lib, pool, q, P.i32([3]), scale=1e-46)
    # the smallest one: all rows alike
    out, lse, _ = P.run_decode(lib, pool, q, P.i32([3]), scale=2.0 ** -149)
    np.testing.assert_allclose(out[0, 0].cpu().numpy(), pool.seq("v", 0)[0].mean(0), atol=1e-5)

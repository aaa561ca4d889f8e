"""Entropies of rows whose logits are so large that a sum of weighted differences of logits
would leave fp32: their scaled differences are of ordinary size."""
import pytest
import torch

from tests import paged_common as P
from tests.test_gpu_logprobs import _run
from tests.test_gpu_logprobs_slices import _check

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [2, 480])
@pytest.mark.parametrize("V", [20000, 128256])
@pytest.mark.parametrize("size", [1e34, 1e35, 1e36, 3e37])
def test_entropy(lib, size, V, n, dtype):
    if n * V > 2e7:
        n = 30
    x = (torch.randn((n, V), device=DEV, generator=P.gen(5)) * size).to(P.DT[dtype])
    x[:, 5::7] = -float("inf")
    tok = P.i32([0] * n)
    r = _run(lib, x, tok, 4, scale=1 / size)
    assert int(r["status"].item()) == 0
    _check(r, x, tok, 4, dtype, scale=1 / size, rows=[0, 1, n - 1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [1e-30, 1e-3, 0.7, 1.0, 1.5, 3.0, 1e3, 1e30, 2.0 ** 127])
def test_masks_beside_every_scale(lib, scale, dtype):
    # masks of minus infinity, of the lowest value and of others far below, at scales whose
    # product with them is finite and not; and logits so large that they are not far below
    V = 20011
    noise = torch.randn((6, V), device=DEV, generator=P.gen(6)) / scale
    x = noise.to(P.DT[dtype])
    low = torch.finfo(x.dtype).min
    x[0, 1::3] = -float("inf")
    x[1, 1::3] = low
    x[2, 1::3] = low
    x[2, 2::5] = -float("inf")
    x[3, 1::3] = -1e37
    x[4] = low / 4
    x[4, ::7] = low
    x[5] = low
    x[5, ::2] = -float("inf")
    tok = P.i32([0, 0, 0, 0, 1, 1])
    r = _run(lib, x, tok, 4, scale=scale)
    assert int(r["status"].item()) == 0
    rows = [i for i in range(6) if i < 3 or abs(float(x[i, int(tok[i])])) * scale < 3e38]
    _check(r, x, tok, 4, dtype, scale=scale, rows=rows)

"""Logit scales at the ends of fp32: the kernels' exponentials work in base 2, so the scale's
product with log2 e must be a number. And at the ends of Python's floats: 0 stands for the
default, so what fp32 rounds to 0 must not be taken for it."""
import pytest
import torch

from tests.test_paged_host import _decode, _logprobs


@pytest.mark.parametrize("scale", [2.0 ** 127 * (1 + 2.0 ** -23), 2.4e38, 3.4e38])
def test_scales_too_large_are_refused(lib, scale):
    assert _logprobs(lib, scale=scale) == lib.EINVAL
    assert _decode(lib, scale=scale) == lib.EINVAL


@pytest.mark.parametrize("scale", [1e-46, -1e-46, 1e-300, 2.0 ** -150])
def test_scales_that_fp32_rounds_to_0_are_refused(lib, scale):
    with pytest.raises(ValueError, match="scale"):
        lib.ripple_token_logprobs(torch.zeros(1, 3), entropy_out=torch.zeros(1), scale=scale)
    # (the smallest that it holds: refused for its host tensors instead)
    with pytest.raises(ValueError, match="CUDA"):
        lib.ripple_token_logprobs(torch.zeros(1, 3), entropy_out=torch.zeros(1), scale=2.0 ** -149)

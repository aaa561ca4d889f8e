"""Logit scales at the ends of fp32: the kernels' exponentials work in base 2, so the scale's
product with log2 e must be a number."""
import pytest

from tests.test_paged_host import _decode, _logprobs


@pytest.mark.parametrize("scale", [2.0 ** 127 * (1 + 2.0 ** -23), 2.4e38, 3.4e38])
def test_scales_too_large_are_refused(lib, scale):
    assert _logprobs(lib, scale=scale) == lib.EINVAL
    assert _decode(lib, scale=scale) == lib.EINVAL

"""ripple_paged_keep_rows without a GPU: what one thread block moves lies apart from what others do, or
the call is refused."""
import ctypes

import pytest
import torch

from tests.test_paged_host import FAKE
from tests.test_paged_more_host import _desc, _keep, _scales

POOL, SCALES = 40 * 2 * 16 * 128, 40 * 2 * 16  # bytes of _desc's codes, scales
KP, VP, KS, VS = FAKE * 4, FAKE * 8, 1 << 32, 2 << 32


def _keep8(lib, layers):
    """layers: (keys, values, their scales) each."""
    L = len(layers)
    P = ctypes.c_void_p * L
    k, v, ks, vs = zip(*layers)
    s = (lib.PagedScales * L)(*[_scales(lib, k=a, v=b) for a, b in zip(ks, vs)])
    return lib._lib.ripple_paged_keep_rows(ctypes.byref(_desc(lib)), s, L, P(*k), P(*v), P(*[FAKE] * L), 12,
                                           None, 4, FAKE * 5, FAKE * 3, FAKE * 3, None, None)


@pytest.mark.parametrize("layer", [
    (KP, VP, KS, KS), (KP, VP, KS, KS + SCALES - 1), (KP, VP, KP, VS), (KP, VP, VP + POOL - 1, VS),
    (KP, VP, KS, KP + POOL - 1), (KP, VP, KS, VP), (KP, VP, KP - SCALES + 1, VS)])
def test_scales_over_one_another_or_over_the_pages(lib, layer):
    good = (KP * 16, VP * 16, KS * 2 + POOL, VS * 4)
    assert _keep8(lib, [layer]) == lib.EINVAL
    assert _keep8(lib, [good, layer]) == lib.EINVAL


def test_scales_beside_one_another_and_the_pages(lib):
    if torch.cuda.is_available():
        pytest.skip("would launch on addresses that are none")
    for layer in ((KP, VP, KS, VS), (KP, VP, KS, KS + SCALES), (KP, VP, KP + POOL, VP + POOL),
                  (KP, VP, KP - SCALES, KP - 2 * SCALES)):
        assert _keep8(lib, [layer]) == lib.ECUDA  # ends at its launch


LENS = 1 << 26  # two layers of three sequences: 24 bytes; kept: 48 of three lists, starts: 16


@pytest.mark.parametrize("over", [
    dict(lens=LENS, lens_out=LENS + 4), dict(lens=LENS, lens_out=LENS + 20),
    dict(lens=LENS, lens_out=LENS - 12), dict(kept=LENS, lens_out=LENS + 44),
    dict(kept=LENS, lens_out=LENS - 20), dict(kept=LENS, lens_out=LENS),
    dict(starts=LENS, lens_out=LENS + 12), dict(starts=LENS, lens_out=LENS - 20)])
def test_lengths_over_what_other_blocks_read(lib, over):
    assert _keep(lib, **dict(dict(lens=FAKE * 3, kept=FAKE * 5, lens_out=FAKE * 3), **over)) == lib.EINVAL


def test_lengths_beside_what_other_blocks_read(lib):
    if torch.cuda.is_available():
        pytest.skip("would launch on addresses that are none")
    for over in (dict(lens=LENS, lens_out=LENS), dict(lens=LENS, lens_out=LENS + 24),
                 dict(lens=LENS, lens_out=LENS - 24), dict(kept=LENS, lens_out=LENS + 48),
                 dict(starts=LENS, lens_out=LENS + 16), dict(most=0, kept=LENS, lens_out=LENS)):
        assert _keep(lib, **dict(dict(lens=FAKE * 3, kept=FAKE * 5, lens_out=FAKE * 3), **over)) == lib.ECUDA

"""Scores that fp32 holds to whole units only, over pages of 16 and 32 bits: the row that has all the
weight is the output, whatever the scores' rounding is worth."""
import numpy as np
import pytest
import torch

from tests import paged8_common as P8
from tests import paged_common as P
from tests import paged_far_common as F

pytestmark = pytest.mark.gpu
DEV = "cuda"
# what a tree's output, one value times a weight over itself, may be off by: fp32 sums; bf16's roundings
# of the weight (which a score's rounding may leave at other than 1) and of the output
REL = {"f32": 1e-4, "bf16": 2 * 2.0 ** -8 + 1e-4}


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("n,G", [(1, 4), (12, 4), (33, 4)])
@pytest.mark.parametrize("up", [18, 24, 30, 60])
def test_trees(lib, up, n, G, kind):
    d, rows, scale = 128, 60 + n, 2.0 ** up
    pool = P8.any_pool(lib, kind, [rows], 1, d, 16, 41)
    q = P.randn((1, n, G, d), kind, 43 + n)
    out, _, st = P8.run_tree(lib, pool, q, P.i32([rows]), torch.full((1, n), -1, device=DEV), scale=scale)
    clear, want = F.one_hot(q.reshape(n * G, d), pool.seq("k", 0)[0], pool.seq("v", 0)[0], scale)
    got = out.reshape(n * G, d).double().cpu().numpy()[clear]
    assert (np.abs(got - want) <= REL[kind] * np.abs(want)).all()


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("G", [1, 4, 8, 16])
@pytest.mark.parametrize("up", [18, 24, 30, 60])
def test_decode(lib, up, G, kind):
    d, rows, scale = 128, 96, 2.0 ** up
    for width in (0, 8192):  # tables with room for little, and for long caches
        pool = P.Pool(lib, [rows], 1, d, 16, kind, 51, width=width)
        q = P.randn((1, G, d), kind, 53 + G)
        out, _, st = P.run_decode(lib, pool, q, P.i32([rows]), scale=scale)
        clear, want = F.one_hot(q[0], pool.seq("k", 0)[0], pool.seq("v", 0)[0], scale)
        got = out[0].double().cpu().numpy()[clear]
        assert (np.abs(got - want) <= 1e-4 * np.abs(want)).all()

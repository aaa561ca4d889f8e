"""The decode over 8-bit pages where all scores of a head are far from 0, against 64 bits."""
import numpy as np
import pytest

from tests import paged8_common as P8
from tests import paged_common as P
from tests import paged_far_common as F

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("G", [1, 4, 8, 16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("far", [-450, -1000, -5000, 5000])
def test_decode_of_scores_far_from_zero(lib, far, d, G, dtype):
    lens = [1, 40, 700, 0]
    q = F.far_queries((4, G, d), dtype, 11) * (1 if far < 0 else -1)
    scale = abs(far) / (1.5 * d * F.LOG2E)
    for width in (0, 8192):  # tables with room for little, and for long caches
        pool = F.far_pool(lib, lens, d, dtype, 10, width)
        out, lse, st = P.run_decode(lib, pool, q, P.i32(lens), scale=scale)
        assert int(st.item()) == 0
        want, want_lse = P.decode_ref(pool, q, lens, scale)
        got, got_lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
        assert (got[3] == 0).all() and np.isinf(got_lse[3]).all()
        for b in range(3):
            k, v = pool.seq("k", b)[0], np.abs(pool.seq("v", b)[0])
            x = q[b].double().cpu().numpy() @ k.T * scale
            assert (np.abs(x) * F.LOG2E > 0.5 * abs(far)).all()
            w = np.exp(x - x.max(1, keepdims=True))
            size = (w / w.sum(1, keepdims=True)) @ v
            top = np.abs(x).max() * F.LOG2E
            assert (np.abs(got[b] - want[b]) <= F.bound("q8-f32", top, size, want[b])).all(), b
            assert (np.abs(got_lse[b] - want_lse[b]) <= 2.0 ** -21 * top + 1e-4).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("G", [4, 8])
@pytest.mark.parametrize("up", [18, 24, 30, 60])
def test_decode_of_scores_that_fp32_holds_to_many_units(lib, up, G, dtype):
    # scores whose neighbours in fp32 are whole units apart: one row has all the weight
    d, n, scale = 128, 60, 2.0 ** up
    for width in (0, 8192):
        pool = P8.Pool8(lib, [n], 1, d, 16, dtype, 31, spread=0.0, width=width)
        pool.vs.random_(120, 135, generator=P.gen(32))
        q = P.randn((1, G, d), dtype, 33 + G)
        out, _, st = P.run_decode(lib, pool, q, P.i32([n]), scale=scale)
        clear, want = F.one_hot(q[0], pool.seq("k", 0)[0], pool.seq("v", 0)[0], scale)
        got = out[0].double().cpu().numpy()[clear]
        assert (np.abs(got - want) <= 1e-4 * np.abs(want)).all()

"""ripple_paged_decode_attn with block tables that have room for long caches, whatever the
lengths: these take another path than tables with room for little, so what is tested of those
is tested of these too, and the two agree."""
import pytest
import torch

from tests import gpu_common as C
from tests import paged_common as P
from tests.test_gpu_checked import chk  # noqa: F401  (fixture)
from tests.test_gpu_paged_checked import test_paged_calls_checked  # noqa: F401
from tests.test_gpu_paged_decode import (  # noqa: F401
    test_a_page_shared_by_sequences, test_lengths_around_every_edge, test_pages_and_layouts,
    test_rows_behind_the_length_never_count, test_scale_and_strided_queries, test_short_caches,
    test_streams_and_graphs_that_share_a_workspace, test_values_that_are_not_finite)

pytestmark = pytest.mark.gpu
ROOM = 1 << 17  # rows


class LongPool(P.Pool):
    def __init__(self, lib, rows, heads, d, page, *args, **kw):
        super().__init__(lib, rows, heads, d, page, *args, **dict(kw, width=ROOM // page))


@pytest.fixture(autouse=True)
def _long_tables(monkeypatch):
    monkeypatch.setattr(P, "Pool", LongPool)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_bad_lengths_and_pages(lib, dtype):
    H, G, d, lens = 2, 3, 64, [400, 640, 64]
    pool = P.Pool(lib, lens, H, d, 16, dtype, 1400)
    q = P.randn((3, H * G, d), dtype, 1401)
    want, want_lse = P.decode_ref(pool, q, lens)
    # rows behind the table's: not there. The pages between are none either
    out, lse, st = P.run_decode(lib, pool, q, P.i32([400, ROOM + 5, 64]))
    assert int(st.item()) in (lib.EFULL, lib.EBOUNDS)
    C.assert_decode_close(out.cpu().numpy(), want)
    out, lse, st = P.run_decode(lib, pool, q, P.i32([400, -2 ** 31, 64]))
    assert int(st.item()) == 0
    assert (out[1] == 0).all() and (lse[1] == -float("inf")).all()
    C.assert_decode_close(out[::2].cpu().numpy(), want[::2])
    for entry in (-1, pool.n_pages, 2 ** 31 - 1):
        pool.table[1] = entry  # no page at all: as an empty one
        out, lse, st = P.run_decode(lib, pool, q, P.i32(lens))
        assert int(st.item()) == lib.EBOUNDS
        assert (out[1] == 0).all() and (lse[1] == -float("inf")).all()
        C.assert_decode_close(out[::2].cpu().numpy(), want[::2])


@pytest.mark.parametrize("dtype,G,d", [("bf16", 4, 128), ("bf16", 13, 64), ("f32", 8, 64)])
def test_agrees_with_short_tables(lib, dtype, G, d):
    lens = [0, 1, 130, 777, 64, 2000]
    a, b = (cls(lib, lens, 2, d, 16, dtype, 1500) for cls in (LongPool, LongPool.__mro__[1]))
    q = P.randn((len(lens), 2 * G, d), dtype, 1501)
    x, xl, _ = P.run_decode(lib, a, q, P.i32(lens))
    y, yl, _ = P.run_decode(lib, b, q, P.i32(lens))
    # both within the kernels' bound of the same values
    assert float((x - y).abs().max()) <= 2 * C.DECODE_PREC_ATOL
    assert torch.equal(xl == -float("inf"), yl == -float("inf"))

"""ripple_paged_decode_attn against the oracle in 64 bits, to the precision bound of the
contiguous decode (tests/gpu_common.py derives it: 1e-4 for values of unit scale); the log
of the sum to the same bound, since an error of a score is the relative error of its
exponential."""
import numpy as np
import pytest
import torch

from tests import gpu_common as C
from tests import paged_common as P

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _check(pool, q, lens, out, lse, scale=None):
    want, want_lse = P.decode_ref(pool, q, lens, scale)
    C.assert_decode_close(out.cpu().numpy(), want)
    got = lse.cpu().numpy().astype(np.float64)
    empty = np.isinf(want_lse)
    assert (got[empty] == -np.inf).all()
    assert (out.cpu().numpy()[np.asarray(lens) <= 0] == 0).all()
    assert np.abs(got[~empty] - want_lse[~empty]).max(initial=0) <= C.DECODE_PREC_ATOL


EDGES = [0, 1, 2, 7, 8, 9, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 511, 4097]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", [1, 2, 3, 4, 5, 7, 8, 11, 16])
def test_lengths_around_every_edge(lib, G, d, dtype):
    pool = P.Pool(lib, EDGES, 1, d, 16, dtype, 100 + G)
    q = P.randn((len(EDGES), G, d), dtype, 200 + G)
    out, lse, st = P.run_decode(lib, pool, q, P.i32(EDGES))
    assert int(st.item()) == 0
    _check(pool, q, EDGES, out, lse)


@pytest.mark.parametrize("page", [1, 2, 4, 8, 32, 64, 128, 1024])
@pytest.mark.parametrize("layout", ["heads", "rows", "pair"])
@pytest.mark.parametrize("dtype,G,H,d", [("bf16", 4, 3, 128), ("f32", 2, 2, 64)])
def test_pages_and_layouts(lib, page, layout, dtype, G, H, d):
    lens = [0, 1, 40, 700, 129, 2500]
    pool = P.Pool(lib, lens, H, d, page, dtype, 300 + page, layout)
    q = P.randn((len(lens), G * H, d), dtype, 301)
    out, lse, st = P.run_decode(lib, pool, q, P.i32(lens))
    assert int(st.item()) == 0
    _check(pool, q, lens, out, lse)


# tables with room for little, as compressed caches have: clusters of 8, 4, 2 and 1 CTAs a
# group, every number of query heads, warps without blocks
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", [1, 2, 4, 7, 16])
@pytest.mark.parametrize("lens,H", [([1], 1), ([0, 470, 33], 2), ([250, 100, 0, 1, 17, 249], 4),
                                    ([100, 3, 64, 0, 31] * 9, 2), ([60, 0, 16, 1] * 50, 2),
                                    ([8, 0, 5, 1] * 100, 2)])
def test_short_caches(lib, lens, H, G, d, dtype):
    for page in (1, 32):
        pool = P.Pool(lib, lens, H, d, page, dtype, 350 + G)
        q = P.randn((len(lens), G * H, d), dtype, 351)
        out, lse, st = P.run_decode(lib, pool, q, P.i32(lens))
        assert int(st.item()) == 0
        _check(pool, q, lens, out, lse)
        again, lse2, _ = P.run_decode(lib, pool, q, P.i32(lens))
        assert torch.equal(out, again) and torch.equal(lse, lse2)


# few long sequences (split and joined), many short ones, both at once
@pytest.mark.parametrize("lens,H,G,d,dtype", [
    ([70001], 1, 8, 128, "bf16"), ([33333, 5], 2, 4, 64, "bf16"), ([20011], 1, 2, 128, "f32"),
    ([3 + 7 * i for i in range(300)], 2, 4, 128, "bf16"),
    ([30000] + [i % 50 for i in range(200)], 1, 1, 64, "f32"),
    ([9000, 1, 0, 12000, 64, 3000 + 71], 8, 4, 128, "bf16"),
    ([0] * 40 + [5] + [0] * 40, 3, 5, 64, "bf16"), ([0, 0], 2, 2, 128, "f32")])
def test_splits(lib, lens, H, G, d, dtype):
    pool = P.Pool(lib, lens, H, d, 32, dtype, 400 + len(lens))
    q = P.randn((len(lens), G * H, d), dtype, 401) * 1.5
    out, lse, st = P.run_decode(lib, pool, q, P.i32(lens))
    assert int(st.item()) == 0
    _check(pool, q, lens, out, lse)
    again, lse2, _ = P.run_decode(lib, pool, q, P.i32(lens))
    assert torch.equal(out, again) and torch.equal(lse, lse2)


def test_equals_the_contiguous_decode_in_exactness(lib):
    # the same cache in pages and in one piece: both within the precision bound of each other
    B, H, G, d, n = 2, 2, 4, 128, 1500
    pool = P.Pool(lib, [n + 1] * B, H, d, 64, "bf16", 500)
    q = P.randn((B, G * H, d), "bf16", 501)
    kc, vc = (torch.stack([torch.from_numpy(pool.seq(w, b)) for b in range(B)]).bfloat16().to(DEV)
              for w in "kv")
    kn, vn = kc[:, :, n].clone()[None], vc[:, :, n].clone()[None]
    desc = lib.decode_desc(1, B, G * H, H, d)
    tables = lib.DecodeTables([kc], [vc])
    out = torch.empty(1, B, G * H, d, device=DEV)
    ws = torch.empty(lib.ripple_decode_workspace_bytes(desc, [n + 1]), dtype=torch.uint8, device=DEV)
    lib.ripple_decode_attn(desc, q[None].contiguous(), kn, vn, tables, P.i32([n]), out, ws)
    got, _, _ = P.run_decode(lib, pool, q, P.i32([n + 1] * B))
    assert float((got - out[0]).abs().max()) <= C.DECODE_PREC_ATOL


@pytest.mark.parametrize("dtype,G", [("bf16", 4), ("bf16", 8), ("bf16", 16), ("f32", 4)])
def test_rows_behind_the_length_never_count(lib, dtype, G):
    # what lies in the last page behind the length, in other pages and in the places of a
    # shorter sequence is not a number; so is every row of the sequences before in shared memory
    lens = [1, 17, 300, 4000] * 40
    pool = P.Pool(lib, lens, 2, 128, 32, dtype, 600)
    q = P.randn((len(lens), 2 * G, 128), dtype, 601)
    keep = torch.zeros(pool.n_pages, 1, pool.page, 1, dtype=torch.bool, device=DEV)
    for b, n in enumerate(lens):
        for r in range(0, n, pool.page):
            keep[pool.np_table[b, r // pool.page], 0, :min(pool.page, n - r)] = True
    for t in (pool.k, pool.v):
        t.masked_fill_(~keep, float("nan"))
    out, lse, st = P.run_decode(lib, pool, q, P.i32(lens))
    assert int(st.item()) == 0
    pick = [0, 1, 2, 3, 81, 158, 159]
    want, want_lse = P.decode_ref(pool, q, [n if b in pick else 0 for b, n in enumerate(lens)])
    C.assert_decode_close(out[pick].cpu().numpy(), want[pick])
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()


@pytest.mark.parametrize("dtype,G,d", [("bf16", 1, 64), ("bf16", 4, 128), ("bf16", 7, 128),
                                       ("bf16", 16, 64), ("f32", 4, 128), ("f32", 16, 64)])
def test_values_that_are_not_finite(lib, dtype, G, d):
    lens = [700, 700, 700, 700]
    pool = P.Pool(lib, lens, 1, d, 16, dtype, 700)
    q = P.randn((4, G, d), dtype, 701)
    base, base_lse, _ = P.run_decode(lib, pool, q, P.i32(lens))
    inf = float("inf")
    p, s = pool.place(0, 333)
    pool.v[p, 0, s, 5] = inf      # its column is infinite, the others as they were
    pool.v[p, 0, s, 6] = -inf
    p, s = pool.place(1, 699)
    pool.k[p, 0, s, 0] = float("nan")  # every output of the group
    # keys of score -infinity count for nothing: a whole run of them too
    q[2, :, 0] = 1.0
    for r in list(range(40, 640)) + [3]:
        p, s = pool.place(2, r)
        pool.k[p, 0, s] = 0
        pool.k[p, 0, s, 0] = -inf
    out, lse, st = P.run_decode(lib, pool, q, P.i32(lens))
    assert int(st.item()) == 0
    o, b = out.cpu().numpy(), base.cpu().numpy()
    assert (o[0, :, 5] == inf).all() and (o[0, :, 6] == -inf).all()
    rest = [i for i in range(d) if i not in (5, 6)]
    assert np.array_equal(o[0][:, rest], b[0][:, rest])
    assert np.isnan(o[1]).all() and np.isnan(lse[1].cpu().numpy()).all()
    live = [r for r in range(700) if not (40 <= r < 640 or r == 3)]
    k, v = pool.seq("k", 2)[0][live], pool.seq("v", 2)[0][live]
    from oracle import ripple_oracle as O
    from paper_2608_08684_gb300 import synth
    C.assert_decode_close(o[2], O.decode_attention(synth.to_f64(q[2]), k, v, d ** -0.5))
    assert np.array_equal(o[3], b[3])


def test_scale_and_strided_queries(lib):
    lens = [100, 3, 555]
    pool = P.Pool(lib, lens, 2, 64, 16, "bf16", 800)
    wide = P.randn((3, 12, 64 + 8), "bf16", 801)
    q = wide[:, 2:10, 8:]
    out, lse, st = P.run_decode(lib, pool, q, P.i32(lens), scale=0.3)
    _check(pool, q, lens, out, lse, 0.3)


def test_bad_lengths_and_pages(lib):
    H, d = 2, 64
    lens = [40, 64, 64]
    pool = P.Pool(lib, lens, H, d, 16, "bf16", 900)
    q = P.randn((3, 4, d), "bf16", 901)
    # longer than the table: its rows count, the rest is reported
    out, lse, st = P.run_decode(lib, pool, q, P.i32([40, 200, 64]))
    assert int(st.item()) == lib.EFULL
    _check(pool, q, lens, out, lse)
    # negative lengths are idle
    out, lse, st = P.run_decode(lib, pool, q, P.i32([40, -5, 64]))
    assert int(st.item()) == 0
    _check(pool, q, [40, 0, 64], out, lse)
    # entries that are no pages: rows left out
    for entry in (-1, pool.n_pages, 2 ** 31 - 1):
        pool.table[1, 2] = entry
        out, lse, st = P.run_decode(lib, pool, q, P.i32(lens))
        assert int(st.item()) == lib.EBOUNDS
        k, v = (pool.seq(w, 1, 64) for w in "kv")
        live = [r for r in range(64) if r // 16 != 2]
        from oracle import ripple_oracle as O
        from paper_2608_08684_gb300 import synth
        for h in range(H):
            ref = O.decode_attention(synth.to_f64(q[1, 2 * h:2 * h + 2]), k[h][live], v[h][live], d ** -0.5)
            C.assert_decode_close(out[1, 2 * h:2 * h + 2].cpu().numpy(), ref)
    pool.table[1] = -1  # no page at all: as an empty one
    out, lse, st = P.run_decode(lib, pool, q, P.i32(lens))
    assert int(st.item()) == lib.EBOUNDS
    assert (out[1] == 0).all() and (lse[1] == -float("inf")).all()


def test_a_page_shared_by_sequences(lib):
    lens = [48, 48]
    pool = P.Pool(lib, lens, 2, 128, 16, "bf16", 1000)
    pool.np_table[1, :2] = pool.np_table[0, :2]  # a shared prefix
    pool.table.copy_(torch.from_numpy(pool.np_table))
    q = P.randn((2, 8, 128), "bf16", 1001)
    out, lse, st = P.run_decode(lib, pool, q, P.i32(lens))
    _check(pool, q, lens, out, lse)


def test_offsets_beyond_32_bits(lib):
    # a pool of 2^31 + elements whose last pages are the sequence's
    H, d, page = 1, 128, 16
    n_pages = (1 << 31) // (page * d) + 40
    k = torch.zeros(n_pages, H, page, d, dtype=torch.bfloat16, device=DEV)
    v = torch.zeros_like(k)
    last = list(range(n_pages - 9, n_pages))
    k[last], v[last] = P.randn((9, H, page, d), "bf16", 1101), P.randn((9, H, page, d), "bf16", 1102)
    pool = P.Pool(lib, [9 * page - 3], H, d, page, "bf16", 1103)
    pool.k, pool.v, pool.n_pages = k, v, n_pages
    pool.np_table = np.array([last], np.int32)
    pool.table = torch.from_numpy(pool.np_table).to(DEV)
    pool.cache = lib.PagedCache(k, v, pool.table)
    q = P.randn((1, 4, d), "bf16", 1104)
    # the last row appended there, then read
    kn, vn = P.randn((1, H, d), "bf16", 1105), P.randn((1, H, d), "bf16", 1106)
    lib.ripple_paged_append(pool.cache, P.i32(pool.rows), kn, vn)
    out, lse, st = P.run_decode(lib, pool, q, P.i32(pool.rows))
    assert torch.equal(v[n_pages - 1, :, 12], vn[0])
    _check(pool, q, pool.rows, out, lse)


def test_streams_and_graphs_that_share_a_workspace(lib):
    lens = [900, 5000]
    pools = [P.Pool(lib, lens, 2, 128, 16, "bf16", 1200 + i) for i in range(2)]
    qs = [P.randn((2, 8, 128), "bf16", 1210 + i) for i in range(2)]
    want = [P.run_decode(lib, p, q, P.i32(lens))[0] for p, q in zip(pools, qs)]
    ws = torch.empty(lib.ripple_paged_decode_workspace_bytes(pools[0].cache, 8), dtype=torch.uint8,
                     device=DEV)
    lens_t = P.i32(lens)
    outs = [torch.zeros(2, 8, 128, device=DEV) for _ in range(2)]
    graphs = []
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for p, q, o in zip(pools, qs, outs):
            lib.ripple_paged_decode_attn(p.cache, q, lens_t, o, ws)
            assert o is not None
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=s):
                lib.ripple_paged_decode_attn(p.cache, q, lens_t, o, ws)
            graphs.append(g)
        for o in outs:
            o.fill_(float("nan"))
        for i in (0, 1, 0, 1, 1, 0):
            graphs[i].replay()
            ws.random_(0, 256)
    s.synchronize()
    for o, w in zip(outs, want):
        assert torch.equal(o, w)
    # a replay reads the lengths of its time
    lens_t.copy_(P.i32([3, 4999]))
    graphs[1].replay()
    torch.cuda.synchronize()
    ref, _ = P.decode_ref(pools[1], qs[1], [3, 4999])
    C.assert_decode_close(outs[1].cpu().numpy(), ref)
    # two at once on two streams, each its own workspace
    ws2 = torch.empty_like(ws)
    lens_t.copy_(P.i32(lens))
    torch.cuda.synchronize()
    s2 = torch.cuda.Stream()
    for _ in range(5):
        with torch.cuda.stream(s):
            lib.ripple_paged_decode_attn(pools[0].cache, qs[0], lens_t, outs[0], ws)
        with torch.cuda.stream(s2):
            lib.ripple_paged_decode_attn(pools[1].cache, qs[1], lens_t, outs[1], ws2)
    torch.cuda.synchronize()
    for o, w in zip(outs, want):
        assert torch.equal(o, w)


def test_binding_refuses_wrong_shapes(lib):
    pool = P.Pool(lib, [4, 4], 2, 64, 8, "f32", 1300)
    q, out = torch.zeros(2, 4, 64, device=DEV), torch.zeros(2, 4, 64, device=DEV)
    ws = torch.empty(lib.ripple_paged_decode_workspace_bytes(pool.cache, 4), dtype=torch.uint8, device=DEV)
    good = dict(q=q, lens=P.i32([4, 4]), out=out, workspace=ws)
    bad = [dict(q=q[:1]), dict(q=q.bfloat16()), dict(q=q[:, :, :32]), dict(out=out.bfloat16()),
           dict(out=out[:, :2]), dict(lse=torch.zeros(2, 3, device=DEV)), dict(lens=P.i32([4])),
           dict(lens=P.i32([4, 4]).long()), dict(q=q.cpu()), dict(out=out.cpu()),
           dict(out=torch.zeros(2, 64, 4, device=DEV).transpose(1, 2))]
    before = lib.ripple_kernel_launches()
    for over in bad:
        with pytest.raises(ValueError):
            lib.ripple_paged_decode_attn(pool.cache, **dict(good, **over))
    with pytest.raises(lib.RippleError) as e:
        lib.ripple_paged_decode_attn(pool.cache, **dict(good, workspace=ws[:128]))
    assert e.value.status == lib.EWORKSPACE
    assert lib.ripple_kernel_launches() == before

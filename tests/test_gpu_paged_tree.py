"""ripple_paged_tree_attn against attention in 64 bits over the rows that each token sees.

fp32 queries: the bound of the decode (1e-4 for values of unit scale, also of the log of the
sum). bf16 queries: a probability is rounded to bf16 (2^-8 of it at most), so the output is
off by 2^-8 sum(p |v|), then rounded, 2^-8 of itself; the log of the sum as in fp32."""
import numpy as np
import pytest
import torch

from tests import gpu_common as C
from tests import paged8_common as P8
from tests import paged_common as P

pytestmark = pytest.mark.gpu
DEV = "cuda"
KINDS = ["bf16", "f32", "q8-bf16", "q8-f32"]


def _check(pool, kind, q, lens, counts, masks, out, lse, scale=None, missing=()):
    Hq, d = q.shape[-2:]
    q = q.reshape(-1, Hq, d)[:sum(counts)]
    want, want_lse, size = P8.tree_ref(pool, q, lens, counts, masks, scale, missing)
    got = out.double().cpu().numpy().reshape(-1, Hq, d)[:len(want)]
    got_lse = lse.double().cpu().numpy().reshape(-1, Hq)[:len(want)]
    unit = max(1.0, float(np.abs(want).max(initial=0.0)))
    bound = C.DECODE_PREC_ATOL * unit
    if P8.type_of(kind) == "bf16":
        bound = bound + 2.0 ** -8 * (size + np.abs(want))
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), (int(bad.sum()), float(np.abs(got - want)[bad].max()))
    empty = np.isinf(want_lse)
    assert (got_lse[empty] == -np.inf).all() and (got[empty] == 0).all()
    assert np.abs(got_lse[~empty] - want_lse[~empty]).max(initial=0) <= C.DECODE_PREC_ATOL


def _ragged(lib, kind, lens, counts, H, G, d, page, seed, layout="heads", masks="tree", width=0,
            max_tokens=None):
    pool = P8.any_pool(lib, kind, [max(0, n) for n in lens], H, d, page, seed, layout)
    n = sum(counts)
    q = P.randn((n + 3, H * G, d), P8.type_of(kind), seed + 50)
    starts = P.i32([0] + np.cumsum(counts).tolist())
    bits = P8.random_masks(counts, seed) if masks == "tree" else masks
    m = None if bits is None else P8.to_i64(bits + [0] * 3)
    out, lse, st = P8.run_tree(lib, pool, q, P.i32(lens), m, starts, max_tokens or max(counts + [1]))
    assert int(st.item()) == 0
    _check(pool, kind, q, lens, counts, bits, out, lse)
    assert torch.isnan(out[n:]).all() and torch.isnan(lse[n:]).all()  # left alone
    return pool, q, out, lse


# rows before the draft around a block's edges, drafts of every size among them
COUNTS = [1, 2, 3, 5, 8, 13, 31, 32, 33, 63, 64, 1, 7, 0, 4, 64, 2]
BEFORE = [0, 1, 31, 32, 33, 59, 60, 63, 64, 65, 127, 128, 200, 9, 1000, 0, 4095]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", [1, 3, 4, 8, 16])
def test_lengths_around_every_edge(lib, G, d, kind):
    lens = [b + n for b, n in zip(BEFORE, COUNTS)]
    _ragged(lib, kind, lens, COUNTS, 1, G, d, 16, 100 + G)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("page", [1, 2, 8, 32, 64, 1024])
@pytest.mark.parametrize("layout", ["heads", "rows"])
def test_pages_and_layouts(lib, page, layout, kind):
    _ragged(lib, kind, [7, 0, 300, 64, 2500, 1], [7, 3, 20, 64, 5, 1], 3, 4, 128, page, 200 + page, layout)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("lens,counts,H,G,d", [
    ([70001], [3], 1, 8, 128), ([33333, 5], [64, 5], 2, 4, 64),
    ([3 + 7 * i for i in range(300)], [1 + i % 3 for i in range(300)], 2, 4, 128),
    ([20000] + [9 + i % 50 for i in range(200)], [64] + [i % 9 for i in range(200)], 1, 2, 64),
    ([9000, 1, 0, 12000, 64], [9, 1, 4, 30, 64], 8, 4, 128),
    ([0] * 40 + [5] + [0] * 40, [2] * 81, 3, 5, 64), ([0, -4], [2, 1], 2, 2, 128),
    ([8000, 4000], [64, 17], 2, 16, 128)])
def test_splits(lib, lens, counts, H, G, d, kind):
    pool, q, out, lse = _ragged(lib, kind, lens, counts, H, G, d, 32, 300 + len(lens))
    starts = P.i32([0] + np.cumsum(counts).tolist())
    bits = P8.to_i64(P8.random_masks(counts, 300 + len(lens)) + [0] * 3)
    again, lse2, _ = P8.run_tree(lib, pool, q, P.i32(lens), bits, starts, max(counts))
    n = sum(counts)
    assert torch.equal(out[:n], again[:n]) and torch.equal(lse[:n], lse2[:n])


# (sequences, KV heads, pages of 32 rows in the table): a group's rows by one team to sixteen, of a
# block each or of eight, with and without an even number of groups, and by runs
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("B,H,pages", [
    (1, 1, 1), (1, 1, 2), (1, 1, 4), (1, 1, 9), (1, 1, 31), (1, 1, 256), (1, 1, 257), (3, 1, 40),
    (19, 1, 33), (20, 1, 130), (19, 2, 16), (13, 3, 64), (38, 2, 7), (7, 11, 33), (76, 2, 4),
    (77, 2, 16), (51, 3, 17), (152, 2, 3), (61, 5, 3), (2, 8, 1024)])
def test_room_of_the_table(lib, B, H, pages, kind):
    rng = np.random.default_rng(B * 1000 + pages)
    G, d, rows = 2, 64, min(pages * 32, 5000)
    counts = [int(n) for n in rng.integers(1, min(rows, 9) + 1, B)]
    lens = [int(n) for n in rng.integers(0, rows + 1, B)]
    lens = [rows if i == 0 else max(n, c) for i, (n, c) in enumerate(zip(lens, counts))]
    if B > 4:
        lens[3] = 0
        counts[3] = 2
    pool = P8.any_pool(lib, kind, lens, H, d, 32, 350 + B, width=pages)
    assert pool.np_table.shape[1] == pages
    q = P.randn((sum(counts), H * G, d), P8.type_of(kind), 351)
    bits = P8.random_masks(counts, 352)
    starts = P.i32([0] + np.cumsum(counts).tolist())
    out, lse, st = P8.run_tree(lib, pool, q, P.i32(lens), P8.to_i64(bits), starts, max(counts))
    assert int(st.item()) == 0
    _check(pool, kind, q, lens, counts, bits, out, lse)
    again, lse2, _ = P8.run_tree(lib, pool, q, P.i32(lens), P8.to_i64(bits), starts, max(counts))
    assert torch.equal(out, again) and torch.equal(lse, lse2)


@pytest.mark.parametrize("kind", KINDS)
def test_uniform_chains_and_strides(lib, kind):
    B, n, H, G, d = 5, 6, 2, 4, 128
    lens = [6, 40, 0, 131, 700]
    pool = P8.any_pool(lib, kind, lens, H, d, 16, 400)
    wide = P.randn((B, n, H * G + 3, d + 8), P8.type_of(kind), 401)
    q = wide[:, :, 1:H * G + 1, 8:]
    out, lse, st = P8.run_tree(lib, pool, q, P.i32(lens), scale=0.21)
    assert int(st.item()) == 0
    _check(pool, kind, q, lens, [n] * B, None, out, lse, 0.21)
    # a chain's mask written out is the same
    bits = P8.to_i64([(1 << (i + 1)) - 1 for _ in range(B) for i in range(n)]).view(B, n)
    out2, lse2, _ = P8.run_tree(lib, pool, q, P.i32(lens), bits, scale=0.21)
    assert torch.equal(out, out2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("kind", KINDS)
def test_one_token_is_the_decode(lib, kind):
    lens = [0, 1, 300, 2000]
    pool = P8.any_pool(lib, kind, lens, 2, 128, 16, 450)
    q = P.randn((4, 8, 128), P8.type_of(kind), 451)
    out, lse, _ = P8.run_tree(lib, pool, q[:, None].contiguous(), P.i32(lens))
    dec, dec_lse, _ = P.run_decode(lib, pool, q, P.i32(lens))
    err = (out[:, 0].double() - dec.double()).abs().max() / max(1.0, float(dec.abs().max()))
    assert float(err) <= (2.0 ** -6 if P8.type_of(kind) == "bf16" else 2 * C.DECODE_PREC_ATOL)
    live = torch.isfinite(dec_lse)
    assert torch.equal(live, torch.isfinite(lse[:, 0]))
    assert float((lse[:, 0] - dec_lse)[live].abs().max()) <= 2 * C.DECODE_PREC_ATOL


@pytest.mark.parametrize("kind", KINDS)
def test_masks_that_leave_nothing(lib, kind):
    counts, lens = [4, 4, 64], [4, 70, 64]
    bits = [0, 1, 0, 5] + [0, 0, 0, 0] + [0] * 63 + [1 << 63]
    _ragged(lib, kind, lens, counts, 2, 4, 64, 16, 500, masks=bits)
    # bits of tokens that are not there
    _ragged(lib, kind, lens, counts, 2, 4, 64, 16, 501, masks=[(1 << 64) - 1] * 72)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("G,before", [(4, 0), (4, 100), (16, 61), (1, 640)])
def test_hidden_rows_count_for_nothing(lib, kind, G, before):
    # drafted tokens whose keys or values are not finite: those that do not see them are as if
    # they were not there, and those that do are infinite or NaN as the sum is
    n, H, d = 12, 1, 128
    bits = P8.random_masks([n], 7)
    bits = [m & ~(1 << 5 | 1 << 7) | (1 << i) for i, m in enumerate(bits)]
    bits[9] |= 1 << 5
    bits[10] |= 1 << 7
    pool = P8.any_pool(lib, kind, [before + n], H, d, 16, 600)
    q = P.randn((1, n, G, d), P8.type_of(kind), 601)
    m = P8.to_i64(bits).view(1, n)
    base, base_lse, _ = P8.run_tree(lib, pool, q, P.i32([before + n]), m)
    p5, s5 = pool.place(0, before + 5)
    p7, s7 = pool.place(0, before + 7)
    if kind.startswith("q8"):
        pool.vs[p5, 0, s5] = 255
        pool.ks[p7, 0, s7] = 255
    else:
        pool.v[p5, 0, s5, 3] = float("inf")
        pool.v[p5, 0, s5, 90] = float("-inf")
        pool.v[p5, 0, s5, 91] = float("nan")
        pool.k[p7, 0, s7, 2] = float("nan")
    out, lse, st = P8.run_tree(lib, pool, q, P.i32([before + n]), m)
    assert int(st.item()) == 0
    sees5, sees7 = ([i for i in range(n) if bits[i] >> j & 1] for j in (5, 7))
    rest = [i for i in range(n) if i not in sees5 and i not in sees7]
    assert len(rest) >= 8
    assert torch.equal(out[0, rest], base[0, rest]) and torch.equal(lse[0, rest], base_lse[0, rest])
    assert torch.isnan(out[0, sees7]).all() and torch.isnan(lse[0, sees7]).all()
    only5 = [i for i in sees5 if i not in sees7]
    assert torch.equal(lse[0, only5], base_lse[0, only5])
    if kind.startswith("q8"):
        assert torch.isnan(out[0, only5]).all()
    else:
        o = out[0, only5].float()
        assert (o[..., 3] == float("inf")).all() and (o[..., 90] == float("-inf")).all()
        assert torch.isnan(o[..., 91]).all()
        cols = [c for c in range(d) if c not in (3, 90, 91)]
        assert torch.equal(o[..., cols], base[0, only5].float()[..., cols])


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_values_before_the_draft_that_are_not_finite(lib, kind):
    n, d, G = 3, 64, 4
    pool = P8.any_pool(lib, kind, [200 + n], 1, d, 16, 620)
    q = P.randn((1, n, G, d), kind, 621)
    base, _, _ = P8.run_tree(lib, pool, q, P.i32([200 + n]))
    p, s = pool.place(0, 150)
    pool.v[p, 0, s, 5] = float("inf")
    out, lse, _ = P8.run_tree(lib, pool, q, P.i32([200 + n]))
    assert (out[0, :, :, 5] == float("inf")).all()
    cols = [c for c in range(d) if c != 5]
    assert torch.equal(out[..., cols], base[..., cols])


@pytest.mark.parametrize("kind", ["q8-bf16", "q8-f32"])
@pytest.mark.parametrize("G,before", [(2, 0), (4, 300), (16, 61)])
def test_scores_below_the_range(lib, G, before, kind):
    # keys of 2^-118 and queries of 2^-80 (and of 0): every score is 0 to fp32, hidden rows stay hidden
    n, H, d = 10, 1, 128
    pool = P8.any_pool(lib, kind, [before + n], H, d, 16, 630)
    pool.ks.fill_(7)
    q = P.randn((1, n, G, d), "f32", 631) * 2.0 ** -80
    q[0, 3] = 0
    q = q.to(P.DT[P8.type_of(kind)])
    bits = P8.random_masks([n], 8)
    out, lse, st = P8.run_tree(lib, pool, q, P.i32([before + n]), P8.to_i64(bits).view(1, n))
    assert int(st.item()) == 0
    _check(pool, kind, q, [before + n], [n], bits, out, lse)


@pytest.mark.parametrize("kind", KINDS)
def test_rows_behind_the_length_never_count(lib, kind):
    lens = [1, 17, 300, 4000] * 10
    counts = [1, 5, 9, 2] * 10
    pool = P8.any_pool(lib, kind, lens, 2, 128, 32, 640)
    keep = torch.zeros(pool.n_pages, 1, pool.page, dtype=torch.bool, device=DEV)
    for b, n in enumerate(lens):
        for r in range(0, n, pool.page):
            keep[pool.np_table[b, r // pool.page], 0, :min(pool.page, n - r)] = True
    for t in (pool.k, pool.v):
        t.masked_fill_(~keep[..., None], 0x7f if kind.startswith("q8") else float("nan"))
    if kind.startswith("q8"):
        for t in (pool.ks, pool.vs):
            t.masked_fill_(~keep, 255)
    n = sum(counts)
    q = P.randn((n, 8, 128), P8.type_of(kind), 641)
    bits = P8.random_masks(counts, 3)
    out, lse, st = P8.run_tree(lib, pool, q, P.i32(lens), P8.to_i64(bits),
                               P.i32([0] + np.cumsum(counts).tolist()), 9)
    assert int(st.item()) == 0
    _check(pool, kind, q, lens, counts, bits, out, lse)


@pytest.mark.parametrize("kind", KINDS)
def test_bad_lengths_starts_and_pages(lib, kind):
    H, G, d = 2, 2, 64
    lens, n = [40, 64, 64], 4
    pool = P8.any_pool(lib, kind, lens, H, d, 16, 700)
    q = P.randn((3, n, H * G, d), P8.type_of(kind), 701)
    # longer than the table: the draft lies behind it, and is left out
    out, lse, st = P8.run_tree(lib, pool, q, P.i32([40, 200, 64]))
    assert int(st.item()) == lib.EFULL
    k, v = pool.seq("k", 1, 64), pool.seq("v", 1, 64)
    for h in range(H):
        x = q[1, :, h * G:(h + 1) * G].double().cpu().numpy() @ k[h].T * d ** -0.5
        w = np.exp(x - x.max(-1, keepdims=True))
        w /= w.sum(-1, keepdims=True)
        got = out[1, :, h * G:(h + 1) * G].double().cpu().numpy()
        assert (np.abs(got - w @ v[h]) <= 1e-3 + 2.0 ** -7 * (w @ np.abs(v[h]))).all()
    # a draft of more tokens than rows: those without a row are left out
    out, lse, st = P8.run_tree(lib, pool, q, P.i32([40, 2, 64]))
    assert int(st.item()) == lib.EBOUNDS
    assert (out[1, :2] == 0).all() and torch.isinf(lse[1, :2]).all()
    assert torch.isfinite(out).all() and torch.isfinite(lse[1, 2:]).all()
    # an entry that is no page
    good = int(pool.table[1, 2])
    for entry in (-1, pool.n_pages, 2 ** 31 - 1):
        pool.table[1, 2] = entry
        out, lse, st = P8.run_tree(lib, pool, q, P.i32(lens))
        assert int(st.item()) == lib.EBOUNDS
        pool.table[1, 2] = good
        _check(pool, kind, q, lens, [n] * 3, None, out, lse,
               missing={(1, r) for r in range(32, 48)})
    pool.table[1] = -1
    out, lse, st = P8.run_tree(lib, pool, q, P.i32(lens))
    assert int(st.item()) == lib.EBOUNDS
    assert (out[1] == 0).all() and (lse[1] == -float("inf")).all()
    pool.table[1] = torch.from_numpy(pool.np_table[1]).to(DEV)
    # starts: more tokens than max_tokens, descending, behind the tensor
    flat = q.reshape(12, H * G, d)
    for starts in ([0, 9, 10, 12], [0, 4, 2, 6], [0, 4, 8, 13], [-1, 2, 4, 6]):
        out, lse, st = P8.run_tree(lib, pool, flat, P.i32(lens), None, P.i32(starts), 5)
        assert int(st.item()) == lib.EBOUNDS, starts


def test_offsets_beyond_32_bits(lib):
    H, d, page = 1, 128, 64
    for kind, size in (("bf16", 1 << 31), ("q8-bf16", 1 << 32)):
        n_pages = size // (page * d) + 20
        rows = 9 * page - 3
        pool = P8.any_pool(lib, kind, [rows], H, d, page, 800)
        small = {x: getattr(pool, x) for x in ("k", "v", "ks", "vs") if hasattr(pool, x)}
        last = list(range(n_pages - 9, n_pages))
        at = torch.from_numpy(pool.np_table[0].astype(np.int64)).to(DEV)
        for x, t in small.items():
            big = torch.zeros((n_pages,) + t.shape[1:], dtype=t.dtype, device=DEV)
            big[last] = t[at]
            setattr(pool, x, big)
        pool.n_pages = n_pages
        pool.np_table = np.array([last], np.int32)
        pool.table = torch.from_numpy(pool.np_table).to(DEV)
        if kind == "bf16":
            pool.cache = lib.PagedCache(pool.k, pool.v, pool.table)
        else:
            pool.bind()
        q = P.randn((1, 5, 4, d), "bf16", 801)
        out, lse, st = P8.run_tree(lib, pool, q, P.i32([rows]))
        assert int(st.item()) == 0
        _check(pool, kind, q, [rows], [5], None, out, lse)


@pytest.mark.parametrize("kind", ["bf16", "q8-bf16", "f32"])
def test_streams_and_graphs_that_share_a_workspace(lib, kind):
    lens, counts = [900, 5000], [6, 11]
    pools = [P8.any_pool(lib, kind, lens, 2, 128, 16, 900 + i) for i in range(2)]
    qs = [P.randn((17, 8, 128), P8.type_of(kind), 910 + i) for i in range(2)]
    starts, lens_t = P.i32([0, 6, 17]), P.i32(lens)
    want = [P8.run_tree(lib, p, q, lens_t, None, starts, 11)[0] for p, q in zip(pools, qs)]
    ws = torch.empty(lib.ripple_paged_tree_workspace_bytes(pools[0].cache, 8, 11), dtype=torch.uint8,
                     device=DEV)
    outs = [torch.zeros_like(q) for q in qs]
    graphs = []
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for p, q, o in zip(pools, qs, outs):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=s):
                lib.ripple_paged_tree_attn(p.cache, q, lens_t, o, ws, seq_starts=starts, max_tokens=11)
            graphs.append(g)
        for o in outs:
            o.fill_(float("nan"))
        for i in (0, 1, 0, 1, 1, 0):
            graphs[i].replay()
            ws.random_(0, 256)
    s.synchronize()
    for o, w in zip(outs, want):
        assert torch.equal(o, w)
    lens_t.copy_(P.i32([30, 4999]))  # a replay reads the lengths and starts of its time
    starts.copy_(P.i32([0, 11, 17]))
    graphs[1].replay()
    torch.cuda.synchronize()
    lse = P8.run_tree(lib, pools[1], qs[1], lens_t, None, starts, 11)[1]
    _check(pools[1], kind, qs[1], [30, 4999], [11, 6], None, outs[1], lse)
    # two at once on two streams, each its own workspace
    ws2 = torch.empty_like(ws)
    lens_t.copy_(P.i32(lens))
    starts.copy_(P.i32([0, 6, 17]))
    torch.cuda.synchronize()
    s2 = torch.cuda.Stream()
    for _ in range(5):
        for st_, i, w in ((s, 0, ws), (s2, 1, ws2)):
            with torch.cuda.stream(st_):
                lib.ripple_paged_tree_attn(pools[i].cache, qs[i], lens_t, outs[i], w,
                                           seq_starts=starts, max_tokens=11)
    torch.cuda.synchronize()
    for o, w in zip(outs, want):
        assert torch.equal(o, w)


@pytest.mark.parametrize("kind", KINDS)
def test_no_tokens(lib, kind):
    pool = P8.any_pool(lib, kind, [8, 8], 2, 64, 8, 1290)
    ws = torch.empty(lib.ripple_paged_tree_workspace_bytes(pool.cache, 4, 3), dtype=torch.uint8, device=DEV)
    before = lib.ripple_kernel_launches()
    for shape, starts in (((2, 0, 4, 64), None), ((0, 4, 64), P.i32([0, 0, 0]))):
        q = torch.zeros(shape, dtype=P.DT[P8.type_of(kind)], device=DEV)
        lib.ripple_paged_tree_attn(pool.cache, q, P.i32([8, 8]), torch.empty_like(q), ws, seq_starts=starts,
                                   max_tokens=None if starts is None else 3)
    assert lib.ripple_kernel_launches() == before


def test_binding_refuses_wrong_shapes(lib):
    pool = P.Pool(lib, [8, 8], 2, 64, 8, "f32", 1300)
    q, out = torch.zeros(2, 3, 4, 64, device=DEV), torch.zeros(2, 3, 4, 64, device=DEV)
    ws = torch.empty(lib.ripple_paged_tree_workspace_bytes(pool.cache, 4, 3), dtype=torch.uint8, device=DEV)
    good = dict(q=q, lens=P.i32([8, 8]), out=out, workspace=ws)
    masks = torch.zeros(2, 3, dtype=torch.int64, device=DEV)
    lib.ripple_paged_tree_attn(pool.cache, **good, masks=masks)
    bad = [dict(q=q[:1]), dict(q=q.bfloat16()), dict(q=q[..., :32]), dict(out=out.bfloat16()),
           dict(out=out[:, :2]), dict(lse=torch.zeros(2, 4, device=DEV)), dict(lens=P.i32([4])),
           dict(lens=P.i32([4, 4]).long()), dict(q=q.cpu()), dict(out=out.cpu()),
           dict(q=q[:, 0], out=out[:, 0]), dict(masks=masks.int()), dict(masks=masks[:1]),
           dict(masks=masks.cpu()), dict(max_tokens=65), dict(seq_starts=P.i32([0, 3, 6])),
           dict(q=q.flatten(0, 1), out=out.flatten(0, 1), seq_starts=P.i32([0, 6]))]
    before = lib.ripple_kernel_launches()
    for over in bad:
        with pytest.raises(ValueError):
            lib.ripple_paged_tree_attn(pool.cache, **dict(good, **over))
    for over, status in ((dict(workspace=ws[:128]), lib.EWORKSPACE), (dict(max_tokens=2), lib.EINVAL),
                         (dict(max_tokens=0), lib.EINVAL)):
        with pytest.raises(lib.RippleError) as e:
            lib.ripple_paged_tree_attn(pool.cache, **dict(good, **over))
        assert e.value.status == status
    assert lib.ripple_kernel_launches() == before

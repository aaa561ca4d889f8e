"""8-bit paged caches: what the append stores against the definition, and the decode over it
against attention in 64 bits over the values that the rows stand for.

A stored row: the fp32 value that is quantised is off by D = 2^-22 (|a| + |b|) of a rotated pair at
most (tests/test_gpu_paged_append.py), nothing otherwise. A code is off by half a step of what
it rounds, 2^-4 of it or 2^-10 below 2^-6; so |code s - x| <= s max(2^-4 |x| / s, 2^-10) + (1 + 2^-4) D.
The decode: its scores lose 2^-22 relative (an fp32 query's two fp16 parts), its
probabilities 2^-22, as much as fp32 sums of these lengths do: the bound of the bf16 cache's
decode, 1e-4 for values of unit scale, holds."""
import numpy as np
import pytest
import torch

from oracle import ripple_oracle as O
from paper_2608_08684_gb300 import synth
from tests import gpu_common as C
from tests import paged8_common as P8
from tests import paged_common as P

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _inv_freq(rot, base=500000.0):
    return [base ** (-2.0 * j / rot) for j in range(rot // 2)]


# dtype, query heads, KV heads, d, page, rot, interleaved, layout, gap, old rows, new tokens, ragged
CASES = [
    ("bf16", 8, 2, 128, 16, 128, False, "heads", 0, [5, 0, 15, 16, 300], [1] * 5, False),
    ("bf16", 4, 4, 64, 8, 64, True, "rows", 0, [0, 7, 8], [3] * 3, False),
    ("bf16", 3, 1, 128, 32, 64, False, "heads", 16, [31, 2, 0, 100], [40, 0, 1, 67], True),
    ("f32", 6, 3, 64, 1, 32, True, "heads", 0, [0, 3], [1, 9], True),
    ("f32", 14, 2, 128, 64, 16, False, "rows", 32, [1, 63, 64, 0, 5, 9], [1, 1, 2, 130, 0, 0], True),
    ("f32", 2, 2, 128, 1024, 128, True, "heads", 0, [2000], [5], False),
    ("bf16", 0, 2, 128, 16, 128, False, "heads", 0, [3, 9], [1, 1], False),
    ("bf16", 8, 2, 64, 16, 0, False, "heads", 0, [3, 9], [4, 4], False),
    ("bf16", 32, 8, 128, 16, 128, False, "heads", 0, [i * 3 for i in range(70)], [1] * 70, False),
    ("f32", 1, 1, 64, 16, 64, False, "rows", 0, [i % 5 for i in range(1100)],
     [i % 3 for i in range(1100)], True),
    ("bf16", 32, 8, 128, 64, 128, False, "heads", 0, [7, 900], [1500, 2500], True),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{c[0]}-{c[1]}q{c[2]}kv-d{c[3]}-p{c[4]}-r{c[5]}")
def test_append_stores_the_definition(lib, case):
    dtype, Hq, H, d, page, rot, inter, layout, gap, old, new, ragged = case
    B, n = len(old), sum(new)
    rows = [o + m for o, m in zip(old, new)]
    pool = P8.Pool8(lib, rows, H, d, page, dtype, 11, layout, gap)
    before = [x.clone() for x in (pool.k, pool.v, pool.ks, pool.vs)]
    pad, first = (5, 2) if ragged else (0, 0)
    room = first + n + pad
    qkv = P.randn((room, Hq + 2 * H, d), dtype, 12)
    qkv *= torch.exp2(4 * torch.randn(room, Hq + 2 * H, 1, device=DEV, generator=P.gen(14))).to(qkv.dtype)
    q, k, v = qkv.split([Hq, H, H], dim=1)
    q_out = P.randn((room, Hq, d), dtype, 13)
    plain = P.Pool(lib, rows, H, d, page, dtype, 11)  # the queries are those of the other call
    q_plain = q_out.clone()
    starts = np.concatenate([[first], first + np.cumsum(new)])
    at = [b for b in range(B) for _ in range(new[b])]
    row = [old[b] + i for b in range(B) for i in range(new[b])]
    pos = [3 * r + 1 for r in row]
    kw = {"positions": P.i32([0] * first + pos + [0] * pad)}
    inv = _inv_freq(rot) if rot else []
    if rot:
        kw["rope"] = lib.Rope(inv, interleaved=inter)
    args = [k, v]
    outs = {}
    if Hq:
        kw["q"] = q
        outs = {"q_out": q_out}, {"q_out": q_plain}
    else:
        outs = {}, {}
    if ragged:
        kw["seq_starts"] = P.i32(starts.tolist())
    else:
        cut = lambda x: x.unflatten(0, (B, new[0]))  # noqa: E731
        args = [cut(x) for x in args]
        kw = {key: cut(x) if key in ("q", "positions") else x for key, x in kw.items()}
        outs = [{key: cut(x) for key, x in o.items()} for o in outs]
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    lib.ripple_paged_append(pool.cache, P.i32(rows), *args, dev_status=status, **kw, **outs[0])
    lib.ripple_paged_append(plain.cache, P.i32(rows), *args, dev_status=status, **kw, **outs[1])
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    if Hq:
        assert torch.equal(q_out, q_plain)
    page_of, slot_of = zip(*[pool.place(b, r) for b, r in zip(at, row)])
    pi, si = torch.tensor(page_of, device=DEV), torch.tensor(slot_of, device=DEV)
    live = slice(first, first + n)
    # values, and keys that are not rotated: byte for byte
    for codes, scales, x in ((pool.v, pool.vs, v), (pool.k, pool.ks, k)):
        got = codes[pi, :, si].view(torch.float8_e4m3fn).double().cpu().numpy()
        byte = scales[pi, :, si].cpu().numpy()
        x64 = synth.to_f64(x[live])
        if codes is pool.v or not rot:
            want, want_byte = P8.quantise64(x64)
            assert np.array_equal(byte, want_byte) and np.array_equal(got, want)
            continue
        want = O.rotate(x64, pos, inv, inter)
        size = O.rotate(np.abs(x64), np.zeros(n), inv, inter)
        half = np.arange(rot // 2)
        one, two = (2 * half, 2 * half + 1) if inter else (half, half + rot // 2)
        D = np.zeros_like(want)
        D[..., one] = D[..., two] = 2.0 ** -22 * (size[..., one] + size[..., two])
        s = np.exp2(byte.astype(np.float64) - 127)[..., None]
        a, most = np.abs(want).max(-1), D.max(-1)
        assert (byte >= 7).all() and (byte <= 247).all()
        assert (a - most <= 448 * s[..., 0]).all()          # the least e that holds the row
        assert ((byte == 7) | (a + most > 224 * s[..., 0])).all()
        bound = np.maximum(2.0 ** -4 * np.abs(want), 2.0 ** -10 * s) + (1 + 2.0 ** -4) * D
        assert (np.abs(got * s - want) <= bound).all()
    # everything else as it was
    for now, was in zip((pool.k, pool.v, pool.ks, pool.vs), before):
        now = now.clone()
        now[pi, :, si] = was[pi, :, si]
        assert torch.equal(now, was)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_append_of_odd_rows(lib, d, dtype):
    # zeros, one value, the borders of the scales, subnormals, the largest, and rows that are not finite
    H, inf, nan = 2, float("inf"), float("nan")
    tops = [0.0, 1.0, 448.0, 449.0 if dtype == "f32" else 450.0, 224.0, 225.0, 2.0 ** -140,
            448 * 2.0 ** -121, 448 * 2.0 ** -120, 449 * 2.0 ** -120 if dtype == "f32" else 450 * 2.0 ** -120,
            3.3e38, 1.875 * 2.0 ** 127, 1.5 * 2.0 ** 127, inf, -inf, nan]
    n = len(tops)
    x = torch.zeros(n, H, d, dtype=torch.float64)
    for i, t in enumerate(tops):
        x[i] = torch.linspace(-0.99, 0.99, d, dtype=torch.float64) * (t if np.isfinite(t) else 2.0)
        x[i, :, 3] = t
        x[i, 1, 5] = -t if t == t else 1.0
    x = x.to(P.DT[dtype]).to(DEV)
    pool = P8.Pool8(lib, [n], H, d, 8, dtype, 21, fill=False)
    lib.ripple_paged_append(pool.cache, P.i32([n]), x[None], x.flip(0)[None])
    for codes, scales, y in ((pool.k, pool.ks, x), (pool.v, pool.vs, x.flip(0))):
        for r in range(n):
            p, s = pool.place(0, r)
            want, byte = P8.quantise64(synth.to_f64(y[r]))
            assert scales[p, :, s].tolist() == byte.tolist(), tops[r]
            got = codes[p, :, s].view(torch.float8_e4m3fn).double().cpu().numpy()
            assert np.array_equal(got, want), tops[r]
            assert (codes[p, :, s][scales[p, :, s] == 255] == 0).all()


def _check(pool, q, lens, out, lse, scale=None):
    want, want_lse = P.decode_ref(pool, q, lens, scale)
    C.assert_decode_close(out.cpu().numpy(), want)
    got = lse.cpu().numpy().astype(np.float64)
    empty = np.isinf(want_lse)
    assert (got[empty] == -np.inf).all()
    assert (out.cpu().numpy()[np.asarray(lens) <= 0] == 0).all()
    assert np.abs(got[~empty] - want_lse[~empty]).max(initial=0) <= C.DECODE_PREC_ATOL


EDGES = [0, 1, 2, 15, 16, 17, 31, 32, 33, 47, 48, 63, 64, 65, 127, 128, 129, 255, 257, 511, 4097]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", [1, 2, 3, 4, 5, 8, 11, 16])
def test_decode_lengths_around_every_edge(lib, G, d, dtype):
    pool = P8.Pool8(lib, EDGES, 1, d, 16, dtype, 100 + G, spread=0.5)
    q = P.randn((len(EDGES), G, d), dtype, 200 + G)
    out, lse, st = P.run_decode(lib, pool, q, P.i32(EDGES))
    assert int(st.item()) == 0
    _check(pool, q, EDGES, out, lse)


@pytest.mark.parametrize("page", [1, 2, 8, 32, 64, 1024])
@pytest.mark.parametrize("layout,gap", [("heads", 0), ("rows", 0), ("heads", 48)])
@pytest.mark.parametrize("dtype,G,H,d", [("bf16", 4, 3, 128), ("f32", 2, 2, 64)])
def test_decode_pages_and_layouts(lib, page, layout, gap, dtype, G, H, d):
    lens = [0, 1, 40, 700, 129, 2500]
    pool = P8.Pool8(lib, lens, H, d, page, dtype, 300 + page, layout, gap, spread=0.5)
    q = P.randn((len(lens), G * H, d), dtype, 301)
    out, lse, st = P.run_decode(lib, pool, q, P.i32(lens))
    assert int(st.item()) == 0
    _check(pool, q, lens, out, lse)


@pytest.mark.parametrize("lens,H,G,d,dtype", [
    ([70001], 1, 8, 128, "bf16"), ([33333, 5], 2, 4, 64, "bf16"), ([20011], 1, 2, 128, "f32"),
    ([3 + 7 * i for i in range(300)], 2, 4, 128, "bf16"),
    ([30000] + [i % 50 for i in range(200)], 1, 16, 64, "f32"),
    ([9000, 1, 0, 12000, 64, 3000 + 71], 8, 4, 128, "bf16"),
    ([0] * 40 + [5] + [0] * 40, 3, 5, 64, "bf16"), ([0, 0], 2, 2, 128, "f32")])
def test_decode_splits(lib, lens, H, G, d, dtype):
    for width in (0, 8192):  # tables with room for little, and for long caches
        pool = P8.Pool8(lib, lens, H, d, 32, dtype, 400 + len(lens), spread=0.3, width=width)
        q = P.randn((len(lens), G * H, d), dtype, 401) * 1.5
        out, lse, st = P.run_decode(lib, pool, q, P.i32(lens))
        assert int(st.item()) == 0
        _check(pool, q, lens, out, lse)
        again, lse2, _ = P.run_decode(lib, pool, q, P.i32(lens))
        assert torch.equal(out, again) and torch.equal(lse, lse2)


@pytest.mark.parametrize("dtype,G,d", [("bf16", 4, 128), ("f32", 8, 64)])
def test_decode_of_very_different_scales(lib, dtype, G, d):
    # rows whose sizes are many powers of two apart: each output to its own size
    n = 500
    pool = P8.Pool8(lib, [n] * 4, 1, d, 16, dtype, 500, spread=0.0)
    q = P.randn((4, G, d), dtype, 501)
    rng = np.random.default_rng(5)
    for b, (ke, ve) in enumerate([(0, 40), (0, -100), (3, 8), (-8, 60)]):
        for r in range(n):
            p, s = pool.place(b, r)
            pool.vs[p, 0, s] = int(np.clip(127 + rng.integers(-abs(ve), abs(ve) + 1), 7, 247))
            pool.ks[p, 0, s] = pool.ks[p, 0, s] + int(rng.integers(min(ke, 0), max(ke, 0) + 1)) // 2
    out, lse, st = P.run_decode(lib, pool, q, P.i32([n] * 4))
    assert int(st.item()) == 0
    got = out.double().cpu().numpy()
    for b in range(4):
        k, v = pool.seq("k", b), pool.seq("v", b)
        x = synth.to_f64(q[b]) @ k[0].T * d ** -0.5
        w = np.exp(x - x.max(1, keepdims=True))
        w /= w.sum(1, keepdims=True)
        # an error of a score is the relative one of its term: 2^-20 of scores of a hundred
        bound = 1e-4 * (w @ np.abs(v[0]))
        assert (np.abs(got[b] - w @ v[0]) <= bound).all(), b


def test_decode_of_huge_and_tiny_queries(lib):
    d, G, n = 128, 4, 300
    pool = P8.Pool8(lib, [n] * 3, 1, d, 16, "bf16", 550, spread=0.0)
    base = P.randn((1, G, d), "bf16", 551)
    q = torch.cat([base * 2.0 ** 40, base, base * 2.0 ** -40])
    for scale, b in ((2.0 ** -43, 0), (0.125, 1), (2.0 ** 37, 2)):
        out, lse, _ = P.run_decode(lib, pool, q, P.i32([n] * 3), scale=scale)
        k, v = pool.seq("k", b), pool.seq("v", b)
        want = O.decode_attention(synth.to_f64(q[b]), k[0], v[0], scale)
        C.assert_decode_close(out[b].cpu().numpy(), want)
    q = torch.zeros(3, G, d, dtype=torch.bfloat16, device=DEV)  # a mean
    out, lse, _ = P.run_decode(lib, pool, q, P.i32([n] * 3))
    assert np.abs(lse.cpu().numpy() - np.log(n)).max() < 1e-5
    C.assert_decode_close(out[1].cpu().numpy(), np.repeat(pool.seq("v", 1)[0].mean(0)[None], G, 0))


@pytest.mark.parametrize("dtype,G", [("bf16", 4), ("bf16", 8), ("bf16", 16), ("f32", 4)])
def test_decode_rows_that_do_not_count(lib, dtype, G):
    # behind the length, in other pages: scales of NaN, codes of NaN
    lens = [1, 17, 300, 4000] * 40
    pool = P8.Pool8(lib, lens, 2, 128, 32, dtype, 600, spread=0.2)
    q = P.randn((len(lens), 2 * G, 128), dtype, 601)
    keep = torch.zeros(pool.n_pages, 1, pool.page, dtype=torch.bool, device=DEV)
    for b, n in enumerate(lens):
        for r in range(0, n, pool.page):
            keep[pool.np_table[b, r // pool.page], 0, :min(pool.page, n - r)] = True
    for t in (pool.k, pool.v):
        t.masked_fill_(~keep[..., None], 0x7f)
    for t in (pool.ks, pool.vs):
        t.masked_fill_(~keep, 255)
    out, lse, st = P.run_decode(lib, pool, q, P.i32(lens))
    assert int(st.item()) == 0
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()
    pick = [0, 1, 2, 3, 81, 158, 159]
    want, _ = P.decode_ref(pool, q, [n if b in pick else 0 for b, n in enumerate(lens)])
    C.assert_decode_close(out[pick].cpu().numpy(), want[pick])


@pytest.mark.parametrize("dtype,G,d", [("bf16", 1, 64), ("bf16", 7, 128), ("f32", 4, 128)])
def test_decode_of_rows_held_as_nan(lib, dtype, G, d):
    lens = [700, 700, 700]
    pool = P8.Pool8(lib, lens, 1, d, 16, dtype, 700, spread=0.2)
    q = P.randn((3, G, d), dtype, 701)
    base, base_lse, _ = P.run_decode(lib, pool, q, P.i32(lens))
    p, s = pool.place(0, 333)
    pool.vs[p, 0, s] = 255   # outputs, not the sums
    p, s = pool.place(1, 699)
    pool.ks[p, 0, s] = 255   # both
    out, lse, st = P.run_decode(lib, pool, q, P.i32(lens))
    assert int(st.item()) == 0
    assert torch.isnan(out[:2]).all() and torch.isnan(lse[1]).all()
    assert torch.equal(lse[0], base_lse[0])
    assert torch.equal(out[2], base[2]) and torch.equal(lse[2], base_lse[2])


def test_decode_scale_and_strided_queries(lib):
    lens = [100, 3, 555]
    pool = P8.Pool8(lib, lens, 2, 64, 16, "bf16", 800, spread=0.3)
    wide = P.randn((3, 12, 64 + 8), "bf16", 801)
    q = wide[:, 2:10, 8:]
    out, lse, st = P.run_decode(lib, pool, q, P.i32(lens), scale=0.3)
    _check(pool, q, lens, out, lse, 0.3)


def test_bad_lengths_and_pages(lib):
    H, d = 2, 64
    lens = [40, 64, 64]
    pool = P8.Pool8(lib, lens, H, d, 16, "bf16", 900, spread=0.2)
    q = P.randn((3, 4, d), "bf16", 901)
    out, lse, st = P.run_decode(lib, pool, q, P.i32([40, 200, 64]))
    assert int(st.item()) == lib.EFULL
    _check(pool, q, lens, out, lse)
    out, lse, st = P.run_decode(lib, pool, q, P.i32([40, -5, 64]))
    assert int(st.item()) == 0
    _check(pool, q, [40, 0, 64], out, lse)
    for entry in (-1, pool.n_pages, 2 ** 31 - 1):
        pool.table[1, 2] = entry
        out, lse, st = P.run_decode(lib, pool, q, P.i32(lens))
        assert int(st.item()) == lib.EBOUNDS
        k, v = (pool.seq(w, 1, 64) for w in "kv")
        live = [r for r in range(64) if r // 16 != 2]
        for h in range(H):
            ref = O.decode_attention(synth.to_f64(q[1, 2 * h:2 * h + 2]), k[h][live], v[h][live], d ** -0.5)
            C.assert_decode_close(out[1, 2 * h:2 * h + 2].cpu().numpy(), ref)
        # nothing is stored there, the scales neither; a row behind the table as well
        was = [x.clone() for x in (pool.k, pool.v, pool.ks, pool.vs)]
        for n, code in ((40, lib.EBOUNDS), (65, lib.EFULL)):
            st.zero_()
            x = P.randn((3, H, d), "bf16", 902)
            lib.ripple_paged_append(pool.cache, P.i32([0, n, 0]), x, x, dev_status=st)
            assert int(st.item()) == code
        assert all(torch.equal(a, b) for a, b in zip(was, (pool.k, pool.v, pool.ks, pool.vs)))


def test_offsets_beyond_32_bits(lib):
    H, d, page = 1, 128, 16
    n_pages = (1 << 32) // (page * d) + 40
    pool = P8.Pool8(lib, [9 * page - 3], H, d, page, "bf16", 1103)
    pool.k = torch.zeros(n_pages, H, page, d, dtype=torch.uint8, device=DEV)
    pool.v = torch.zeros_like(pool.k)
    pool.ks = torch.full((n_pages, H, page), 127, dtype=torch.uint8, device=DEV)
    pool.vs = pool.ks.clone()
    pool.n_pages = n_pages
    last = list(range(n_pages - 9, n_pages))
    pool.np_table = np.array([last], np.int32)
    pool.table = torch.from_numpy(pool.np_table).to(DEV)
    pool.bind()
    kn, vn = P.randn((1, 9 * page - 3, H, d), "bf16", 1105), P.randn((1, 9 * page - 3, H, d), "bf16", 1106)
    lib.ripple_paged_append(pool.cache, P.i32(pool.rows), kn, vn)
    q = P.randn((1, 4, d), "bf16", 1104)
    out, lse, st = P.run_decode(lib, pool, q, P.i32(pool.rows))
    want, _ = P8.quantise64(synth.to_f64(vn[0, -1]))
    assert np.array_equal(pool.v[n_pages - 1, :, 12].view(torch.float8_e4m3fn).double().cpu().numpy(), want)
    _check(pool, q, pool.rows, out, lse)


def test_streams_and_graphs_that_share_a_workspace(lib):
    lens = [900, 5000]
    pools = [P8.Pool8(lib, lens, 2, 128, 16, "bf16", 1200 + i, spread=0.2) for i in range(2)]
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
    lens_t.copy_(P.i32([3, 4999]))
    graphs[1].replay()
    torch.cuda.synchronize()
    ref, _ = P.decode_ref(pools[1], qs[1], [3, 4999])
    C.assert_decode_close(outs[1].cpu().numpy(), ref)


def test_scales_without_a_place_for_every_row_are_refused(lib):
    pool = P8.Pool8(lib, [20, 20], 2, 64, 8, "bf16", 990)
    f8, e8 = torch.float8_e4m3fn, torch.float8_e8m0fnu
    one = torch.full((1, 1, 1), 127, dtype=torch.uint8, device=DEV).expand(pool.ks.shape).view(e8)
    with pytest.raises(ValueError):  # (strides of 0 alone mean dense ones to the C call)
        lib.PagedCache(pool.k.view(f8), pool.v.view(f8), pool.table, k_scales=one, v_scales=one)

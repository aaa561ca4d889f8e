"""Trees over 8-bit pages whose rows have scales far apart, rows that are hidden or have no weight, and
scores far from 0, against 64 bits."""
import numpy as np
import pytest
import torch

from tests import paged8_common as P8
from tests import paged_common as P
from tests import paged_far_common as F

pytestmark = pytest.mark.gpu
DEV = "cuda"
KINDS = ["q8-bf16", "q8-f32"]
# tokens and heads: four copies of the query rows, two, one, several tiles
SHAPES = [(4, 4), (8, 4), (12, 4), (30, 4), (64, 5)]


@pytest.mark.parametrize("kind", ["q8-bf16", "q8-f32"])
@pytest.mark.parametrize("n,G", [(3, 1), (8, 4), (12, 4), (33, 4)])
@pytest.mark.parametrize("far", [-450, -1000, -5000, 5000])
def test_trees_of_scores_far_from_zero(lib, far, n, G, kind):
    d, dtype = 128, P8.type_of(kind)
    lens = [n, n + 40, 700]
    q = F.far_queries((3, n, G, d), dtype, 21) * (1 if far < 0 else -1)
    scale = abs(far) / (1.5 * d * F.LOG2E)
    bits = P8.random_masks([n] * 3, 22)
    for width in (0, 8192):
        pool = F.far_pool(lib, lens, d, dtype, 20, width)
        out, lse, st = P8.run_tree(lib, pool, q, P.i32(lens), P8.to_i64(bits).view(3, n), scale=scale)
        assert int(st.item()) == 0
        flat = q.reshape(3 * n, G, d)
        want, want_lse, size = P8.tree_ref(pool, flat, lens, [n] * 3, bits, scale)
        top = 1.5 * abs(far)
        got = out.double().cpu().numpy().reshape(want.shape)
        assert (np.abs(got - want) <= F.bound(kind, top, size, want)).all()
        err = np.abs(lse.double().cpu().numpy().reshape(want_lse.shape) - want_lse)
        assert (err <= 2.0 ** -21 * top + 1e-4).all()


@pytest.mark.parametrize("kind", ["q8-bf16", "q8-f32"])
@pytest.mark.parametrize("n,G", [(1, 4), (12, 4), (33, 4)])
@pytest.mark.parametrize("up", [18, 24, 30, 60])
def test_trees_of_scores_that_fp32_holds_to_many_units(lib, up, n, G, kind):
    d, rows, scale = 128, 60 + n, 2.0 ** up
    pool = P8.Pool8(lib, [rows], 1, d, 16, P8.type_of(kind), 41, spread=0.0)
    pool.vs.random_(120, 135, generator=P.gen(42))
    q = P.randn((1, n, G, d), P8.type_of(kind), 43 + n)
    out, _, st = P8.run_tree(lib, pool, q, P.i32([rows]), torch.full((1, n), -1, device=DEV), scale=scale)
    clear, want = F.one_hot(q.reshape(n * G, d), pool.seq("k", 0)[0], pool.seq("v", 0)[0], scale)
    got = out.reshape(n * G, d).double().cpu().numpy()[clear]
    rel = 1e-4 if kind == "q8-f32" else 2.0 ** -8 + 2.0 ** -11 + 1e-4
    assert (np.abs(got - want) <= rel * np.abs(want)).all()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n,G", SHAPES)
@pytest.mark.parametrize("before", [0, 50, 700])
def test_hidden_rows_of_any_scale_count_for_nothing(lib, before, n, G, kind):
    d, hide = 128, [0, n // 2]
    bits = [m & ~sum(1 << j for j in hide) | 1 << i for i, m in enumerate(P8.random_masks([n], 51))]
    for i, j in enumerate(hide):  # each seen by itself alone
        bits[j] = 1 << j
    pool = P8.any_pool(lib, kind, [before + n], 1, d, 16, 52)
    q = P.randn((1, n, G, d), P8.type_of(kind), 53)
    m = P8.to_i64(bits).view(1, n)
    base, base_lse, _ = P8.run_tree(lib, pool, q, P.i32([before + n]), m)
    rest = [i for i in range(n) if i not in hide]
    for byte in (137, 152, 170, 247, 7):
        for which in (pool.ks, pool.vs):
            was = which.clone()
            for j in hide:
                p, s = pool.place(0, before + j)
                which[p, 0, s] = byte
            out, lse, st = P8.run_tree(lib, pool, q, P.i32([before + n]), m)
            which.copy_(was)
            assert int(st.item()) == 0
            assert torch.equal(out[0, rest], base[0, rest]), byte
            assert torch.equal(lse[0, rest], base_lse[0, rest]), byte


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n,G", SHAPES)
@pytest.mark.parametrize("up", [20, 40, 100])
def test_rows_without_weight_take_nothing_from_the_others(lib, up, n, G, kind):
    # before the draft and in it: keys with all scores far below, values 2^up (then 2^(2 up)) larger
    d, dtype, rows = 128, P8.type_of(kind), 150 + n
    pool = P8.any_pool(lib, kind, [rows], 1, d, 16, 61)
    q = F.far_queries((1, n, G, d), dtype, 62)
    bits = [0] + [m | 1 for m in P8.random_masks([n], 63)[1:]]
    far = [3, 66, 140, 150]  # (150: the draft's first token, seen by all others)
    for low in (False, True):  # all other values tiny
        pool.vs.fill_(127 - (up if low else 0))
        pool.ks.fill_(120)
        p, s = (x[far] for x in F.rows(pool, 0, rows))
        pool.k[p, 0, s] = F.codes(-torch.ones(len(far), d))
        pool.ks[p, 0, s] = 134  # a score of about -128 sqrt(d) log2(e)
        pool.vs[p, 0, s] = 127 + up
        out, lse, st = P8.run_tree(lib, pool, q, P.i32([rows]), P8.to_i64(bits).view(1, n))
        assert int(st.item()) == 0
        flat = q.reshape(n, G, d)
        want, want_lse, size = P8.tree_ref(pool, flat, [rows], [n], bits)
        got = out[0].double().cpu().numpy()
        assert (np.abs(got - want) <= F.bound(kind, 64.0, size, want)).all()
        assert np.abs(lse[0].double().cpu().numpy() - want_lse).max() <= 1e-4 + 2.0 ** -21 * 64


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n,G", SHAPES)
@pytest.mark.parametrize("ke,ve", [(0, 40), (0, -100), (3, 8), (-8, 60)])
def test_scales_far_apart(lib, ke, ve, n, G, kind):
    # rows whose sizes are many powers of two apart: each output to its own size
    d, rows = 128, [400 + n, n, 2000]
    pool = P8.any_pool(lib, kind, rows, 1, d, 16, 71)
    rng = np.random.default_rng(72)
    shape = tuple(pool.vs.shape)
    pool.vs.copy_(torch.from_numpy(127 + rng.integers(-abs(ve), abs(ve) + 1, shape)).to(DEV))
    pool.ks.copy_(torch.from_numpy(119 + rng.integers(min(ke, 0), max(ke, 0) + 1, shape) // 2).to(DEV))
    q = P.randn((3, n, G, d), P8.type_of(kind), 73)
    bits = P8.random_masks([n] * 3, 74)
    out, lse, st = P8.run_tree(lib, pool, q, P.i32(rows), P8.to_i64(bits).view(3, n))
    assert int(st.item()) == 0
    flat = q.reshape(3 * n, G, d)
    want, want_lse, size = P8.tree_ref(pool, flat, rows, [n] * 3, bits)
    got = out.double().cpu().numpy().reshape(want.shape)
    assert (np.abs(got - want) <= F.bound(kind, 64.0, size, want)).all()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n,G", [(4, 4), (12, 4), (30, 4)])
def test_keys_of_far_scales_beside_others(lib, n, G, kind):
    # keys 2^100 smaller than their neighbours have scores of 0, not their neighbours' precision; queries
    # that are tiny, so that only the largest keys have scores
    d, rows = 128, 300 + n
    pool = P8.any_pool(lib, kind, [rows], 1, d, 16, 81)
    rng = np.random.default_rng(82)
    far = rng.random(tuple(pool.ks.shape)) < 0.3
    for lo, hi, size in ((19, 119, 1.0), (119, 219, 2.0 ** -100)):
        pool.ks.copy_(torch.from_numpy(np.where(far, hi, lo)).to(DEV))
        q = (P.randn((1, n, G, d), "f32", 83) * size).to(P.DT[P8.type_of(kind)])
        out, lse, st = P8.run_tree(lib, pool, q, P.i32([rows]))
        assert int(st.item()) == 0
        want, want_lse, size64 = P8.tree_ref(pool, q.reshape(n, G, d), [rows], [n], None)
        assert (np.abs(out[0].double().cpu().numpy() - want) <= F.bound(kind, 64.0, size64, want)).all()
        assert np.abs(lse[0].double().cpu().numpy() - want_lse).max() <= 1e-4 + 2.0 ** -21 * 64


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page,layout", [(1, "rows"), (8, "heads"), (64, "rows"), (1024, "heads")])
@pytest.mark.parametrize("G,most", [(2, 16), (4, 16), (7, 64)])
def test_scales_far_apart_among_rows_that_are_none(lib, G, most, page, layout, d, kind):
    # rows of any scale beside hidden rows held as NaN, entries that are no page, rows behind the
    # length; over tables with room for little and for much
    H, rng = 3, np.random.default_rng(page + d)
    counts = [int(n) for n in rng.integers(1, most + 1, 12)]
    rows = [n + int(rng.integers(0, 900)) for n in counts]
    bits = P8.random_masks(counts, 91)
    for width in (0, 8192 // page):
        pool = P8.any_pool(lib, kind, rows, H, d, page, 90, layout, width=width)
        shape = tuple(pool.vs.shape)
        pool.vs.copy_(torch.from_numpy(rng.integers(87, 168, shape)).to(DEV))
        pool.ks.copy_(torch.from_numpy(118 + rng.integers(-30, 2, shape)).to(DEV))
        missing, hide, t0 = set(), [], 0
        masks = list(bits)
        for b, (n, m) in enumerate(zip(rows, counts)):
            if b % 3 == 0 and n - m > 2 * page:  # an entry before the draft
                at = int(rng.integers(0, (n - m) // page - 1))
                pool.table[b, at] = -1
                missing |= {(b, r) for r in range(at * page, min((at + 1) * page, n - m))}
            if m > 2:  # a drafted token that no other sees
                j = int(rng.integers(1, m))
                p, s = pool.place(b, n - m + j)
                (pool.vs if b % 2 else pool.ks)[p, :, s] = 255
                hide.append(t0 + j)
                for i in range(m):
                    masks[t0 + i] &= ~(1 << j)
                masks[t0 + j] |= 1 << j
            t0 += m
        q = P.randn((sum(counts), H * G, d), P8.type_of(kind), 93)
        starts = P.i32([0] + np.cumsum(counts).tolist())
        out, lse, st = P8.run_tree(lib, pool, q, P.i32(rows), P8.to_i64(masks), starts, most)
        assert int(st.item()) == (lib.EBOUNDS if missing else 0)
        want, want_lse, size = P8.tree_ref(pool, q, rows, counts, masks, missing=missing)
        got, got_lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
        rest = [i for i in range(sum(counts)) if i not in hide]
        assert np.isfinite(want[rest]).all()
        assert (np.abs(got - want) <= F.bound(kind, 64.0, size, want))[rest].all()
        assert (np.abs(got_lse - want_lse)[rest] <= 1e-4 + 2.0 ** -21 * 64).all()
        assert np.isnan(got[hide]).all() and (np.isnan(got_lse) == np.isnan(want_lse)).all()

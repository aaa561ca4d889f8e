"""ripple_paged_keep_rows: rows moved bit for bit, everything else as it was, the new lengths."""
import numpy as np
import pytest
import torch

from tests import paged8_common as P8
from tests import paged_common as P

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _tensors(pool):
    return [getattr(pool, x) for x in ("k", "v", "ks", "vs") if hasattr(pool, x)]


def _expect(pools, lens, counts, kept):
    """The tensors after the call, moved on the host, and the lengths."""
    new_lens = np.array(lens)
    out = []
    for l, pool in enumerate(pools):
        ts = [t.cpu().clone() for t in _tensors(pool)]
        for b, n in enumerate(lens[l]):
            if n <= 0:
                continue
            path = []
            for x in kept[b]:
                if x < 0 or x >= counts[b] or (path and x <= path[-1]):
                    break
                path.append(x)
            first = n - counts[b]
            for j, x in enumerate(path):
                (sp, ss), (dp, ds) = pool.place(b, first + x), pool.place(b, first + j)
                for t in ts:
                    t[dp, :, ds] = t[sp, :, ss].clone()
            new_lens[l][b] = first + len(path)
        out.append(ts)
    return out, new_lens


@pytest.mark.parametrize("kind", ["bf16", "f32", "q8-bf16", "q8-f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page,layout,L", [(1, "heads", 1), (16, "rows", 3), (64, "heads", 128)])
@pytest.mark.parametrize("ragged", [False, True])
def test_rows_move(lib, kind, d, page, layout, L, ragged):
    B, H = 6, 3
    counts = [64, 1, 16, 40, 2, 7] if ragged else [9] * B
    rng = np.random.default_rng(L + page)
    lens = [[int(c + rng.integers(0, 70)) for c in counts] for _ in range(L)]
    lens[0][4] = 0     # idle
    pools = [P8.any_pool(lib, kind, lens[l], H, d, page, 10 + l, layout) for l in range(L)]
    width = max(p.table.shape[1] for p in pools)
    n_pages = max(p.n_pages for p in pools)
    for p in pools:  # one shape for all layers
        p.np_table = np.pad(p.np_table, ((0, 0), (0, width - p.np_table.shape[1])), constant_values=-3)
        p.table = torch.from_numpy(p.np_table).to(DEV)
        for x in ("k", "v", "ks", "vs"):
            if hasattr(p, x):
                t = getattr(p, x)
                if layout == "rows":
                    t = torch.cat([t, t[:1].expand(n_pages - p.n_pages, *t.shape[1:])]).transpose(1, 2)
                    t = t.contiguous().transpose(1, 2)
                else:
                    t = torch.cat([t, t[:1].expand(n_pages - p.n_pages, *t.shape[1:])]).contiguous()
                setattr(p, x, t)
        if kind.startswith("q8"):
            p.bind()
        else:
            p.cache = lib.PagedCache(p.k, p.v, p.table)
    kept = [[-1] * 16 for _ in range(B)]
    for b, c in enumerate(counts):
        path = sorted(rng.choice(c, size=rng.integers(0, min(c, 16) + 1), replace=False).tolist())
        kept[b][:len(path)] = path
    kept[0] = list(range(0, 64, 4)) if ragged else kept[0]
    want, want_lens = _expect(pools, lens, counts, kept)
    tables = lib.KeepTables([p.cache for p in pools])
    lens_t = P.i32(lens)
    lens_out = torch.full_like(lens_t, -9)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    kw = dict(seq_starts=P.i32([3] + (3 + np.cumsum(counts)).tolist())) if ragged else dict(n_tokens=9)
    lib.ripple_paged_keep_rows(tables, lens_t, P.i32(kept), lens_out=lens_out, dev_status=st, **kw)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    assert lens_t.tolist() == lens and lens_out.tolist() == want_lens.tolist()
    for p, ts in zip(pools, want):
        assert all(torch.equal(a.cpu(), b) for a, b in zip(_tensors(p), ts))
    # the lengths in place, nothing kept
    lib.ripple_paged_keep_rows(tables, lens_t, P.i32([[]] * B), dev_status=st, **kw)
    assert lens_t.tolist() == [[n - c if n > 0 else n for n, c in zip(row, counts)] for row in lens]
    for p, ts in zip(pools, want):
        assert all(torch.equal(a.cpu(), b) for a, b in zip(_tensors(p), ts))


@pytest.mark.parametrize("kind", ["bf16", "q8-bf16"])
def test_entries_that_are_none(lib, kind):
    lens, n = [[40, 40, 40, 3, 64, 90]], 8
    kept = [[0, 3, 8, -1], [2, 2, 5, -1], [5, 4, 6, 7], [0, 1, -1, -1], [1, 3, -1, -1], [7, -1, 2, 5]]
    pool = P8.any_pool(lib, kind, [40, 40, 40, 8, 64, 64], 2, 64, 16, 50)
    want, want_lens = _expect([pool], [[40, 40, 40, 0, 64, 0]], [n] * 6, kept)
    tables = lib.KeepTables([pool.cache])
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    lens_t = P.i32(lens)
    lib.ripple_paged_keep_rows(tables, lens_t, P.i32(kept), n_tokens=n, dev_status=st)
    # 3: fewer rows than tokens, as it was; 5: rows behind the table (64) are not moved
    assert lens_t.tolist() == [want_lens[0][:3].tolist() + [3, int(want_lens[0][4]), 83]]
    assert int(st.item()) in (lib.EBOUNDS, lib.EFULL)
    assert all(torch.equal(a.cpu(), b) for a, b in zip(_tensors(pool), want[0]))
    # each by itself
    for b, status in ((0, lib.EBOUNDS), (1, lib.EBOUNDS), (2, lib.EBOUNDS), (3, lib.EBOUNDS), (4, 0),
                      (5, lib.EFULL)):
        one = [0] * 6
        one[b] = lens[0][b]
        st.zero_()
        lib.ripple_paged_keep_rows(tables, P.i32([one]), P.i32(kept), n_tokens=n, dev_status=st)
        assert int(st.item()) == status, b
    # a page that is none: its rows stay, the others move
    pool.table[4, 3] = -1  # rows 48 .. 63: the draft
    was = [t.clone() for t in _tensors(pool)]
    st.zero_()
    lens_t = P.i32([[0, 0, 0, 0, 64, 0]])
    lib.ripple_paged_keep_rows(tables, lens_t, P.i32(kept), n_tokens=n, dev_status=st)
    assert int(st.item()) == lib.EBOUNDS and int(lens_t[0, 4]) == 58
    assert all(torch.equal(a, b) for a, b in zip(_tensors(pool), was))


def test_drafts_of_descending_starts_change_nothing(lib):
    pool = P8.any_pool(lib, "bf16", [40, 40, 40], 2, 64, 16, 55)
    tables = lib.KeepTables([pool.cache])
    was = [t.clone() for t in _tensors(pool)]
    for kept in ([[0, -1], [-1, -1], [-1, -1]], [[0, 1], [0, 1], [0, 1]]):
        st, lens_t = torch.zeros(1, dtype=torch.int32, device=DEV), P.i32([[40, 40, 40]])
        lib.ripple_paged_keep_rows(tables, lens_t, P.i32(kept), seq_starts=P.i32([0, 4, 1, 3]),
                                   dev_status=st)
        n = [len([e for e in k if e >= 0]) for k in kept]
        assert lens_t.tolist() == [[36 + n[0], 40, 38 + n[2]]] and int(st.item()) == lib.EBOUNDS
        assert all(torch.equal(a, b) for a, b in zip(_tensors(pool), was))


def test_a_captured_call_reads_what_is_accepted_at_its_time(lib):
    L, n = 2, 6
    lens = [[50, 20], [33, 48]]
    pools = [P.Pool(lib, [64, 64], 2, 128, 16, "bf16", 60 + l) for l in range(L)]
    tables = lib.KeepTables([p.cache for p in pools])
    lens_t, kept = P.i32(lens), P.i32([[-1] * 4] * 2)
    lens_out = torch.zeros_like(lens_t)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        lib.ripple_paged_keep_rows(tables, lens_t, kept, n_tokens=n, lens_out=lens_out)
    for path in ([[0, 2, 4, -1], [1, 3, 4, 5]], [[5, -1, -1, -1], [0, 1, 2, 3]]):
        want, want_lens = _expect(pools, lens, [n] * 2, path)
        kept.copy_(P.i32(path))
        g.replay()
        torch.cuda.synchronize()
        assert lens_out.tolist() == want_lens.tolist()
        for p, ts in zip(pools, want):
            assert all(torch.equal(a.cpu(), b) for a, b in zip(_tensors(p), ts))


def test_binding_refuses_wrong_shapes(lib):
    pools = [P.Pool(lib, [20, 20], 2, 64, 8, "f32", 70 + i) for i in range(2)]
    other = P.Pool(lib, [20, 20], 2, 128, 8, "f32", 75)
    with pytest.raises(ValueError):
        lib.KeepTables([pools[0].cache, other.cache])
    with pytest.raises(ValueError):
        lib.KeepTables([])
    with pytest.raises(ValueError):  # a layer twice: its rows would be moved twice at a time
        lib.KeepTables([pools[0].cache, pools[1].cache, pools[0].cache])
    t = lib.KeepTables([p.cache for p in pools])
    lens, kept = P.i32([[20, 20]] * 2), P.i32([[0, 1]] * 2)
    before = lib.ripple_kernel_launches()
    for args, kw in (((lens[:1], kept), dict(n_tokens=4)), ((lens.long(), kept), dict(n_tokens=4)),
                     ((lens, kept[:1]), dict(n_tokens=4)), ((lens, kept), {}),
                     ((lens, kept), dict(n_tokens=4, seq_starts=P.i32([0, 4, 8]))),
                     ((lens, kept), dict(seq_starts=P.i32([0, 4]))),
                     ((lens.cpu(), kept), dict(n_tokens=4)),
                     ((lens, kept), dict(n_tokens=4, lens_out=lens[0]))):
        with pytest.raises(ValueError):
            lib.ripple_paged_keep_rows(t, *args, **kw)
    with pytest.raises(lib.RippleError):
        lib.ripple_paged_keep_rows(t, lens, P.i32([[0] * 65] * 2), n_tokens=4)
    assert lib.ripple_kernel_launches() == before

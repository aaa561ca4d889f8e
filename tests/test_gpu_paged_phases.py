"""ripple_paged_decode_attn over large batches, whose runs come in three phases: more than 64
groups and more than 32 blocks of 4 KB for every place on the GPU (8 an SM). Lengths far apart
with idle sequences among them, a group that a phase ends within, rows behind a length and
pages of no sequence NaN; against the formula in 64 bits on every sequence."""
import numpy as np
import pytest
import torch

from tests import gpu_common as C
from tests import paged_common as P
from tests.test_gpu_checked import chk  # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu
DEV = "cuda"
ROOM = 1 << 18  # rows of the tables: never the short caches' kernel


def _places():
    return 8 * torch.cuda.get_device_properties(0).multi_processor_count


def _lens(H, B, rb, seed):
    """Rows of every sequence: at least twice the blocks that three phases need, an idle or a
    short one here and there, and a long one that the first phase ends within."""
    rng = np.random.default_rng(seed)
    blocks = 2 * 32 * _places() // H
    kind = np.arange(B) % 8
    share = rng.uniform(0.3, 1.7, B) * (kind > 1)
    share[B * 3 // 4] = share.sum() / 8
    lens = np.ceil(share / share.sum() * blocks * rb).astype(np.int64) - rng.integers(0, rb, B)
    lens[kind == 0] = 0
    lens[kind == 1] = rng.integers(1, 3 * rb, B)[kind == 1]
    lens = np.maximum(lens, 0)
    per = -(-lens // rb)
    starts = np.concatenate([[0], np.cumsum(np.repeat(per, H))])
    total = int(starts[-1])
    assert B * H > 64 and total > 1.9 * 32 * _places() and lens.max() <= ROOM
    for share in (190, 236):  # the phases end within groups
        assert total * share // 256 not in starts
    return lens.tolist()


def _ref(pool, q, lens, drop=None):
    """The formula in 64 bits, on the GPU; rows r of sequence b with drop(b, r) left out."""
    B, Hq, d = q.shape
    G = Hq // pool.heads
    out = torch.zeros(B, Hq, d, dtype=torch.float64, device=DEV)
    lse = torch.full((B, Hq), -float("inf"), dtype=torch.float64, device=DEV)
    for b, n in enumerate(lens):
        if n == 0:
            continue
        pages = torch.from_numpy(pool.np_table[b, :-(-n // pool.page)].astype(np.int64)).to(DEV)
        k, v = (t[pages].transpose(0, 1).reshape(pool.heads, -1, d)[:, :n].double()
                for t in (pool.k, pool.v))
        if drop is not None and drop[0] == b:
            keep = torch.arange(n, device=DEV) // pool.page != drop[1]
            k, v = k[:, keep], v[:, keep]
        for h in range(pool.heads):
            at = slice(h * G, (h + 1) * G)
            x = q[b, at].double() @ k[h].T * d ** -0.5
            m = x.amax(1, keepdim=True)
            w = torch.exp(x - m)
            s = w.sum(1, keepdim=True)
            out[b, at] = w @ v[h] / s
            lse[b, at] = (m + torch.log(s))[:, 0]
    return out.cpu().numpy(), lse.cpu().numpy()


def _pool(lib, lens, H, d, dtype, seed, page=32):
    pool = P.Pool(lib, lens, H, d, page, dtype, seed, width=ROOM // page)
    for t in (pool.k, pool.v):
        t[pool.spare] = float("nan")
        for b, n in enumerate(lens):
            if n % page:
                t[int(pool.np_table[b, n // page]), :, n % page:] = float("nan")
    return pool


def _check(out, lse, want, want_lse):
    C.assert_decode_close(out.cpu().numpy(), want)
    got, empty = lse.cpu().numpy().astype(np.float64), np.isinf(want_lse)
    assert (got[empty] == -np.inf).all() and (out.cpu().numpy()[empty] == 0).all()
    assert np.abs(got[~empty] - want_lse[~empty]).max() <= C.DECODE_PREC_ATOL


CASES = [("bf16", 4, 2, 128, 90), ("bf16", 8, 3, 64, 70), ("bf16", 16, 1, 128, 124),
         ("f32", 1, 2, 128, 90), ("f32", 8, 4, 64, 60), ("f32", 3, 1, 64, 120)]


@pytest.mark.parametrize("dtype,G,H,d,B", CASES)
def test_lengths_far_apart(lib, dtype, G, H, d, B):
    rb = 4096 // (d * (2 if dtype == "bf16" else 4))
    lens = _lens(H, B, rb, G)
    pool = _pool(lib, lens, H, d, dtype, 2000)
    q = P.randn((B, G * H, d), dtype, 2001)
    out, lse, st = P.run_decode(lib, pool, q, P.i32(lens))
    assert int(st.item()) == 0
    _check(out, lse, *_ref(pool, q, lens))
    again, lse2, _ = P.run_decode(lib, pool, q, P.i32(lens))
    assert torch.equal(out, again) and torch.equal(lse, lse2)


@pytest.mark.parametrize("dtype,G,d", [("bf16", 4, 128), ("f32", 2, 64)])
def test_values_that_are_not_finite_and_bad_pages(lib, dtype, G, d):
    H, B = 2, 90
    rb = 4096 // (d * (2 if dtype == "bf16" else 4))
    lens = _lens(H, B, rb, G)
    pool = _pool(lib, lens, H, d, dtype, 2100)
    q = P.randn((B, G * H, d), dtype, 2101)
    base, base_lse, _ = P.run_decode(lib, pool, q, P.i32(lens))
    long = B * 3 // 4
    p, s = pool.place(long, lens[long] - 1)
    pool.k[p, 0, s, 0] = float("nan")               # a whole group
    p, s = pool.place(long - 1, lens[long - 1] // 2)
    pool.v[p, 1, s, 5] = float("inf")               # a column of a group
    gone = lens[long + 1] // pool.page // 2
    pool.table[long + 1, gone] = pool.n_pages       # a page of both groups
    out, lse, st = P.run_decode(lib, pool, q, P.i32(lens))
    assert int(st.item()) == lib.EBOUNDS
    assert torch.isnan(out[long, :G]).all() and torch.isnan(lse[long, :G]).all()
    assert (out[long - 1, G:, 5] == float("inf")).all()
    want, want_lse = _ref(pool, q, [n if b == long + 1 else 0 for b, n in enumerate(lens)],
                          drop=(long + 1, gone))
    _check(out[long + 1:long + 2], lse[long + 1:long + 2], want[long + 1:long + 2],
           want_lse[long + 1:long + 2])
    # nothing else moved
    out[long, :G], lse[long, :G] = base[long, :G], base_lse[long, :G]
    out[long - 1, G:, 5] = base[long - 1, G:, 5]
    out[long + 1], lse[long + 1] = base[long + 1], base_lse[long + 1]
    assert torch.equal(out, base) and torch.equal(lse, base_lse)


@pytest.mark.parametrize("dtype,G,d", [("bf16", 8, 128), ("f32", 4, 64)])
def test_checked(lib, chk, dtype, G, d):  # noqa: F811
    # the bounds-checked build: no access out of range, and the same outputs
    H, B = 2, 90
    rb = 4096 // (d * (2 if dtype == "bf16" else 4))
    lens = _lens(H, B, rb, G)
    q = P.randn((B, G * H, d), dtype, 2201)
    runs = []
    for m in (lib, chk):
        pool = _pool(m, lens, H, d, dtype, 2200)
        runs.append(P.run_decode(m, pool, q, P.i32(lens)))
    assert int(runs[1][2].item()) == 0
    assert torch.equal(runs[0][0], runs[1][0]) and torch.equal(runs[0][1], runs[1][1])

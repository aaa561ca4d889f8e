"""ripple_paged_append against the rotation in 64 bits.

Tolerance of a rotated value a cos - b sin: cosine and sine of an angle exact to 2^-32
turns, its rest rounded to fp32 (2^-28 turns, 2.4e-8), and 1 ulp of the functions (2^-24 for
values up to 1): at most 1e-7 each; the product and the fused multiply-add round by 2^-24 of
their size each. Together below 2^-22 (|a| + |b|); then the one rounding to the cache's type.
Copied values are equal bit for bit, and what no token belongs to is left as it was."""
import numpy as np
import pytest
import torch

from oracle import ripple_oracle as O
from paper_2608_08684_gb300 import synth
from tests import paged_common as P

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _inv_freq(rot, base=500000.0):
    return [base ** (-2.0 * j / rot) for j in range(rot // 2)]


def _check_rotated(got, x, pos, inv, inter, dtype):
    """got, x [n][heads][d] tensors; x turned to pos."""
    want = O.rotate(synth.to_f64(x), pos, inv, inter)
    size = O.rotate(np.abs(synth.to_f64(x)), np.zeros(len(pos)), inv, inter)
    half = len(inv)
    first = np.arange(half) * 2 if inter else np.arange(half)
    second = first + (1 if inter else half)
    pair = np.zeros_like(size)
    pair[..., first] = pair[..., second] = size[..., first] + size[..., second]
    # the rounded value is at most half a step from the computed one
    bound = 2.0 ** -22 * pair
    bound = bound + P.HALF_STEP[dtype] * (np.abs(want) + bound) * (pair > 0)
    err = np.abs(synth.to_f64(got) - want)
    assert (err <= bound).all(), float((err - bound).max())


# dtype, query heads, KV heads, d, page, rot, interleaved, layout, old rows, new tokens, ragged
CASES = [
    ("bf16", 8, 2, 128, 16, 128, False, "heads", [5, 0, 15, 16, 300], [1] * 5, False),
    ("bf16", 4, 4, 64, 8, 64, True, "rows", [0, 7, 8], [3] * 3, False),
    ("bf16", 3, 1, 128, 32, 64, False, "pair", [31, 2, 0, 100], [40, 0, 1, 67], True),
    ("f32", 6, 3, 64, 1, 32, True, "heads", [0, 3], [1, 9], True),
    ("f32", 14, 2, 128, 64, 16, False, "rows", [1, 63, 64, 0, 5, 9], [1, 1, 2, 130, 0, 0], True),
    ("f32", 2, 2, 128, 1024, 128, True, "pair", [2000], [5], False),
    ("bf16", 0, 2, 128, 16, 128, False, "heads", [3, 9], [1, 1], False),       # no queries
    ("bf16", 8, 2, 64, 16, 0, False, "heads", [3, 9], [4, 4], False),          # no rotation
    ("bf16", 32, 8, 128, 16, 128, False, "heads", [i * 3 for i in range(70)], [1] * 70, False),
    ("bf16", 1, 1, 64, 16, 64, False, "rows", [i % 5 for i in range(1100)],
     [i % 3 for i in range(1100)], True),                                      # many sequences
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{c[0]}-{c[1]}q{c[2]}kv-d{c[3]}-p{c[4]}-r{c[5]}")
@pytest.mark.parametrize("positions", ["rows", "given"])
def test_append_matches_the_formula(lib, case, positions):
    dtype, Hq, H, d, page, rot, inter, layout, old, new, ragged = case
    B, n = len(old), sum(new)
    rows = [o + m for o, m in zip(old, new)]
    pool = P.Pool(lib, rows, H, d, page, dtype, 11, layout)
    k0, v0 = pool.k.clone(), pool.v.clone()
    pad = 5 if ragged else 0  # rows behind the last token
    first = 2 if ragged else 0  # and before the first
    room = first + n + pad
    qkv = P.randn((room, Hq + 2 * H, d), dtype, 12)
    q, k, v = qkv.split([Hq, H, H], dim=1)
    q_out = P.randn((room, Hq, d), dtype, 13)
    q_before = q_out.clone()
    starts = np.concatenate([[first], first + np.cumsum(new)])
    at = [b for b in range(B) for _ in range(new[b])]
    row = [old[b] + i for b in range(B) for i in range(new[b])]
    pos = row
    kw = {}
    if positions == "given":
        rng = np.random.default_rng(5)
        pos = rng.integers(0, 200000, n).tolist()
        pos[0] = 2 ** 31 - 1  # far, and negative
        pos[-1] = -12345 if n > 1 else pos[-1]
        kw["positions"] = P.i32([0] * first + pos + [0] * pad)
    inv = _inv_freq(rot) if rot else []
    if rot:
        kw["rope"] = lib.Rope(inv, interleaved=inter)
    args = [k, v]
    if Hq:
        kw.update(q=q, q_out=q_out)
    if ragged:
        kw["seq_starts"] = P.i32(starts.tolist())
    else:
        m = new[0]
        args = [x.unflatten(0, (B, m)) for x in args]
        kw = {key: x.unflatten(0, (B, m)) if key in ("q", "q_out", "positions") else x
              for key, x in kw.items()}
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    lens = P.i32(rows)
    lib.ripple_paged_append(pool.cache, lens, *args, dev_status=status, **kw)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    page_of, slot_of = zip(*[pool.place(b, r) for b, r in zip(at, row)])
    pi, si = torch.tensor(page_of, device=DEV), torch.tensor(slot_of, device=DEV)
    live = slice(first, first + n)
    assert torch.equal(pool.v[pi, :, si], v[live])
    if rot:
        _check_rotated(pool.k[pi, :, si], k[live], pos, inv, inter, dtype)
        assert torch.equal(pool.k[pi, :, si][..., rot:], k[live][..., rot:])
        if Hq:
            _check_rotated(q_out[live], q[live], pos, inv, inter, dtype)
    else:
        assert torch.equal(pool.k[pi, :, si], k[live])
        assert torch.equal(q_out[live], q[live])
    # everything else as it was
    for now, before in ((pool.k, k0), (pool.v, v0)):
        now = now.clone()
        now[pi, :, si] = before[pi, :, si]
        assert torch.equal(now, before)
    if Hq:
        assert torch.equal(q_out[:first], q_before[:first])
        assert torch.equal(q_out[first + n:], q_before[first + n:])


def test_queries_rotate_in_place_and_rows_lie_anywhere(lib):
    # the fused projection's output, its queries turned where they are; heads and tokens far apart
    B, n, Hq, H, d = 3, 2, 4, 2, 128
    pool = P.Pool(lib, [40, 2, 17], H, d, 16, "bf16", 21)
    wide = P.randn((Hq + 2 * H, n, B, d + 24), "bf16", 22)
    qkv = wide[..., 8:8 + d].permute(2, 1, 0, 3)  # [B][n][heads][d]
    q, k, v = qkv.split([Hq, H, H], dim=2)
    before = wide.clone()
    want = q.clone()
    inv = _inv_freq(d)
    pos = P.i32([[7, 8], [0, 1], [100000, 3]])
    lib.ripple_paged_append(pool.cache, P.i32(pool.rows), k, v, rope=lib.Rope(inv), positions=pos,
                            q=q, q_out=q)
    torch.cuda.synchronize()
    _check_rotated(q.reshape(-1, Hq, d), want.reshape(-1, Hq, d), pos.flatten().tolist(), inv, False,
                   "bf16")
    for b in range(B):
        for i in range(n):
            page, slot = pool.place(b, pool.rows[b] - n + i)
            assert torch.equal(pool.v[page, :, slot], v[b, i])
    wide[:Hq, :, :, 8:8 + d] = before[:Hq, :, :, 8:8 + d]
    assert torch.equal(wide, before)  # nothing but the queries


def test_idle_sequences_and_bad_places(lib):
    # idle sequences store nothing and report nothing; rows before the first, entries that
    # are no pages and rows behind the table are not stored, and reported
    H, d = 2, 64
    EFULL, EBOUNDS = lib.EFULL, lib.EBOUNDS
    for lens, new, expect, stored in [
            ([0, 5, -3], 2, 0, [(1, 3), (1, 4)]),
            ([1, 5, 9], 2, EBOUNDS, [(0, 0), (1, 3), (1, 4), (2, 7), (2, 8)]),
            ([33, 5, 9], 2, EFULL, [(0, 31), (1, 3), (1, 4), (2, 7), (2, 8)])]:
        pool = P.Pool(lib, [32, 32, 32], H, d, 8, "f32", 31)
        k0, v0 = pool.k.clone(), pool.v.clone()
        k, v = P.randn((3, new, H, d), "f32", 32), P.randn((3, new, H, d), "f32", 33)
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        lib.ripple_paged_append(pool.cache, P.i32(lens), k, v, dev_status=status)
        torch.cuda.synchronize()
        assert int(status.item()) == expect, lens
        for b, r in stored:
            page, slot = pool.place(b, r)
            i = r - (lens[b] - new)
            assert torch.equal(pool.v[page, :, slot], v[b, i]) and torch.equal(pool.k[page, :, slot], k[b, i])
            pool.k[page, :, slot], pool.v[page, :, slot] = k0[page, :, slot], v0[page, :, slot]
        assert torch.equal(pool.k, k0) and torch.equal(pool.v, v0), lens
    for entry in (-1, 10 ** 6):
        pool = P.Pool(lib, [32, 32, 32], H, d, 8, "f32", 31)
        k0 = pool.k.clone()
        pool.table[1, 1] = entry
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        lib.ripple_paged_append(pool.cache, P.i32([0, 10, 0]), k, v, dev_status=status)
        torch.cuda.synchronize()
        assert int(status.item()) == EBOUNDS and torch.equal(pool.k, k0)


def test_no_tokens(lib):
    pool = P.Pool(lib, [4], 2, 64, 8, "f32", 41)
    before = lib.ripple_kernel_launches()
    empty = torch.empty(0, 2, 64, device=DEV)
    lib.ripple_paged_append(pool.cache, P.i32([4]), empty, empty, seq_starts=P.i32([0, 0]))
    assert lib.ripple_kernel_launches() == before
    k0 = pool.k.clone()
    some = torch.ones(3, 2, 64, device=DEV)
    lib.ripple_paged_append(pool.cache, P.i32([4]), some, some, seq_starts=P.i32([0, 0]))
    torch.cuda.synchronize()
    assert torch.equal(pool.k, k0)


def test_values_that_are_not_finite_are_copied(lib):
    pool = P.Pool(lib, [2, 2], 1, 64, 8, "bf16", 51)
    k, v = P.randn((2, 1, 64), "bf16", 52), P.randn((2, 1, 64), "bf16", 53)
    v[0, 0, :4] = torch.tensor([float("nan"), float("inf"), -float("inf"), -0.0], dtype=torch.bfloat16)
    k[1, 0, 3] = float("inf")
    lib.ripple_paged_append(pool.cache, P.i32([2, 2]), k, v, rope=lib.Rope(_inv_freq(64)),
                            positions=P.i32([5, 1]))
    torch.cuda.synchronize()
    page, slot = pool.place(0, 1)
    assert torch.equal(pool.v[page, 0, slot].view(torch.int16), v[0, 0].view(torch.int16))
    page, slot = pool.place(1, 1)
    hit = ~torch.isfinite(pool.k[page, 0, slot])
    assert hit.nonzero().flatten().tolist() == [3, 35]  # the pair it is in


def test_binding_refuses_wrong_shapes(lib):
    pool = P.Pool(lib, [4, 4], 2, 64, 8, "f32", 61)
    t = lambda *s: torch.zeros(*s, device=DEV)  # noqa: E731
    lens, k = P.i32([4, 4]), t(2, 2, 64)
    bad = [
        dict(k=t(3, 2, 64), v=t(3, 2, 64)), dict(v=t(2, 1, 64)), dict(k=k.bfloat16()),
        dict(k=t(2, 2, 128)[..., ::2]), dict(v=t(2, 2, 2, 64)), dict(q=t(2, 4, 64)),
        dict(q_out=t(2, 4, 64)), dict(q=t(2, 4, 64), q_out=t(2, 1, 4, 64)),
        dict(positions=P.i32([1, 2, 3])), dict(positions=P.i32([1, 2]).long()),
        dict(seq_starts=P.i32([0, 1])), dict(lens=P.i32([4])), dict(lens=lens.long()),
        dict(lens=lens.cpu()), dict(k=k.cpu(), v=k.cpu()), dict(positions=P.i32([1, 2]).cpu()),
    ]
    before = lib.ripple_kernel_launches()
    for over in bad:
        kw = dict(dict(lens=lens, k=k, v=k), **over)
        with pytest.raises(ValueError):
            lib.ripple_paged_append(pool.cache, **kw)
    assert lib.ripple_kernel_launches() == before

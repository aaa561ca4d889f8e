"""ripple_token_logprobs where a row is cut into slices (a cluster of CTAs), and in the
narrow CTAs of many rows, against the oracle in 64 bits.

Tolerances. d = x - max is rounded (2^-24), so is its product with the scale in base 2, which
is itself rounded (2^-24 each): a term's relative error is 2^-22 of the exponential and
3 2^-24 |y| ln 2 of its argument, y in base 2, that is 2^-22.4 |scale d|. Of the sums these are
averages over the terms, computed here. Additions: a thread sums every second of its logits,
V / (64 W slices) of them in a CTA of W warps (32 of a chunk, and 8 of a partial vector, more at
most), and 1 + 5 joins within the warp, 2^-24 each. Larger maxima than the first chunk's
(`moves`), 3 joins of the warps and 3 of the slices rescale a part of the sums: an exponential,
its argument (x exp(-x) <= 0.37), and three roundings, below 2^-21 of the sum each.
log1p(S') is off by the relative error of S' and 2^-22 of its own rounding; log P by
2^-22 |scale d| more; the entropy has log1p(S') and T / (1 + S')."""
import numpy as np
import pytest
import torch

from oracle import ripple_oracle as O
from paper_2608_08684_gb300 import synth
from tests import paged_common as P
from tests.test_gpu_checked import chk  # noqa: F401  (fixture)
from tests.test_gpu_logprobs import _logits, _run

pytestmark = pytest.mark.gpu
DEV = "cuda"
INF = float("inf")
PLACES, CHUNK = 456, 16384  # CTAs at a time, bytes of a CTA's chunk


def _slices(n, V, dtype):
    """How many slices a row of the call is cut into, and the warps of a CTA."""
    size = V * {"bf16": 2, "f32": 4}[dtype]
    c = 1
    while size > 4 * CHUNK and c < 8 and n * 2 * c <= PLACES and size >= 2 * c * CHUNK:
        c *= 2
    return c, 2 if n > PLACES and size <= 128 * 1024 else 8


def _check(r, logits, tokens, top, dtype, scale=1.0, rows=None, moves=8):
    n, V = logits.shape
    slices, W = _slices(n, V, dtype)
    joins = (V / (64 * W * slices) + 32 + 8 + 6) * 2.0 ** -24 + (moves + 3 + 3) * 2.0 ** -21
    h = {k: None if t is None else t.cpu().numpy() for k, t in r.items()}
    scale = float(np.float32(scale))
    for i in range(n) if rows is None else rows:
        x = synth.to_f64(logits[i])
        m = x.max()
        d = np.where(x == -INF, 0.0, scale * (x - m))
        w = np.where(x == -INF, 0.0, np.exp(d))
        w[x.argmax()] = 0
        S, T, Q = w.sum(), -(w * d).sum(), (w * d * d).sum()
        l1, T1 = np.log1p(S), T / (1 + S)
        es = 2.0 ** -22 + (2.0 ** -22.4 * T / S if S > 0 else 0) + joins
        et = 2.0 ** -22 + (2.0 ** -22.4 * Q / T if T > 0 else 0) + 2.0 ** -23 + joins
        lp, _ = O.token_logprobs(x, scale)

        def close(got, t, what):
            if x[t] == -INF:
                assert got == -INF, (what, i, t, got)
                return
            want = d[t] - l1
            # (the oracle subtracts its log of the sum, of the size of the largest logit)
            assert abs(lp[t] - want) <= 2.0 ** -46 * (abs(scale * m) + abs(d[t]) + l1)
            bound = 2.0 ** -22 * abs(d[t]) + (es + 2.0 ** -22) * l1 + 1e-30
            assert abs(got - want) <= bound, (what, i, t, got, want)

        close(h["logprob"][i], int(tokens[i]), "logprob")
        bound = (es + 2.0 ** -22) * l1 + (et + es + 2.0 ** -22) * T1 + 1e-30
        assert abs(h["entropy"][i] - (l1 + T1)) <= bound, (i, h["entropy"][i], l1 + T1)
        bound = (es + 2.0 ** -22) * l1 + 2.0 ** -23 * (abs(scale * m) + l1) + 1e-30
        assert abs(h["lse"][i] - (scale * m + l1)) <= bound, (i, h["lse"][i])
        if top:
            want = O.top_tokens(x, top)
            assert h["idx"][i].tolist() == want.tolist(), (i, h["idx"][i], want)
            for j, t in enumerate(want):
                close(h["top"][i, j], t, "top")


def _tokens(n, V):
    """Tokens of every slice, and the row's ends."""
    return P.i32([(i * 2654435761 % V) if i % 3 else (V - 1 if i % 2 else 0) for i in range(n)])


COUNTS = [1, 57, 58, 114, 115, 153, 228, 229, 457]


@pytest.mark.parametrize("dtype,V", [("bf16", 70001), ("f32", 40001), ("bf16", 40003)])
def test_every_number_of_slices(lib, dtype, V):
    assert {_slices(n, V, dtype)[0] for n in COUNTS} == ({1, 2, 4} if V == 40003 else {1, 2, 4, 8})
    for n in COUNTS:
        x = _logits(n, V, dtype, 700 + n, stride=V + 1, offset=1)
        tok = _tokens(n, V)
        r = _run(lib, x, tok, 20, scale=0.7)
        assert int(r["status"].item()) == 0
        _check(r, x, tok, 20, dtype, scale=0.7, rows=sorted({0, n // 3, n - 2, n - 1} - {-1}))
        again = _run(lib, x, tok, 20, scale=0.7)
        for k in ("logprob", "entropy", "lse", "idx", "top"):
            assert torch.equal(r[k], again[k]), (n, k)


def _slice_start(s, V, dtype, slices):
    """First logit of slice s, for a row that starts at a 16-byte boundary."""
    e = {"bf16": 8, "f32": 4}[dtype]
    return -(-V // e) // slices * s * e


@pytest.mark.parametrize("dtype,V", [("bf16", 70001), ("f32", 40001)])
@pytest.mark.parametrize("n", [12, 100, 200])
@pytest.mark.parametrize("top", [1, 32])
def test_masks_and_ties_over_the_slices(lib, top, n, dtype, V):
    slices = _slices(n, V, dtype)[0]
    assert slices == {12: 8, 100: 4, 200: 2}[n]
    at = lambda s: _slice_start(s, V, dtype, slices)  # noqa: E731
    x = _logits(n, V + (-V % 8), dtype, 800 + n)[:, :V]  # rows start at a 16-byte boundary
    low = torch.finfo(P.DT[dtype]).min
    x[0, :at(slices - 1)] = -INF                       # the last slice alone
    x[1, at(1):] = -INF                                # the first alone
    x[2] = -INF
    x[2, [at(1) - 1, at(1), V - 1]] = torch.tensor([1.0, 1.0, 2.0], device=DEV).to(x.dtype)
    x[3] = 1.5                                         # ties of every slice
    x[4] = 0.0
    x[4, ::3] = -0.0
    x[5] = low / 2                                     # nothing but one huge value
    x[6] = low / 2
    x[6, at(1):] = -INF
    x[7] = torch.arange(V, device=DEV).to(x.dtype) / 4096   # ascending over the slices
    x[8] = -torch.arange(V, device=DEV).to(x.dtype) / 4096  # and descending
    for s in range(slices):                            # the likeliest the last of every slice
        x[9, (at(s + 1) if s + 1 < slices else V) - 1] = 30.0
    x[10, at(1):] = x[10, :V - at(1)].clone()          # the first slice's logits once more
    tok = _tokens(n, V)
    tok[0], tok[2], tok[6] = V - 1, at(1), 5
    r = _run(lib, x, tok, top, scale=1.25)
    assert int(r["status"].item()) == 0
    special = list(range(11))
    # (a row that ascends moves its maximum with every chunk)
    _check(r, x, tok, top, dtype, scale=1.25, rows=special, moves=V // 4096 + 8)
    _check(r, x, tok, top, dtype, scale=1.25, rows=[11, n - 1])


@pytest.mark.parametrize("dtype,V", [("bf16", 70001), ("f32", 40001)])
@pytest.mark.parametrize("n", [12, 100, 200])
def test_rows_without_a_distribution(lib, n, dtype, V):
    slices = _slices(n, V, dtype)[0]
    at = lambda s: _slice_start(s, V, dtype, slices)  # noqa: E731
    x = _logits(n, V + (-V % 8), dtype, 900 + n)[:, :V]
    bad = torch.tensor([float("nan"), INF, -INF], device=DEV).to(x.dtype)
    x[0, at(slices - 1) + 77] = bad[0]
    x[1, at(1)] = bad[1]
    x[2] = -INF
    x[3, :at(1)] = bad[0]                    # nothing but NaN in the first slice
    x[4, at(slices - 1):] = bad[0]
    x[5, V - 1] = bad[0]                     # in the last, partial vector
    x[6] = -INF
    x[6, at(1) + 3] = bad[0]                 # beside masks alone
    x[7, at(1):] = bad[1]
    x[7, 0] = bad[0]                         # both, in different slices
    tok = _tokens(n, V)
    r = _run(lib, x, tok, 32)
    assert int(r["status"].item()) == 0
    for i in range(8):
        assert torch.isnan(r["logprob"][i]) and torch.isnan(r["entropy"][i]), i
        assert torch.isnan(r["top"][i]).all(), i
        idx = r["idx"][i].tolist()
        assert len(set(idx)) == 32 and min(idx) >= 0 and max(idx) < V, i
        assert (r["lse"][i].item() == -INF) if i == 2 else torch.isnan(r["lse"][i]), i
    _check(r, x, tok, 32, dtype, rows=[8, 9, 10, 11, n - 1])


@pytest.mark.parametrize("dtype,V", [("bf16", 70001), ("f32", 40001)])
def test_logits_of_every_size(lib, dtype, V):
    # scales and logits at the type's ends, masks of the lowest value beside infinite ones
    n = 12
    slices = _slices(n, V, dtype)[0]
    low = torch.finfo(P.DT[dtype]).min
    tok = _tokens(n, V)
    for size, scale in ((1e34, 2e-34), (1e32, 2e-32), (1e-30, 1e30), (3.0, 1.0)):
        x = (torch.randn((n, V), device=DEV, generator=P.gen(17)) * size).to(P.DT[dtype])
        x[:, 5::3] = -INF
        if size == 3.0:
            x[:, 7::5] = low
        x[0, :_slice_start(3, V, dtype, slices)] = -INF
        x[1, _slice_start(3, V, dtype, slices):] = low if size == 3.0 else -INF
        r = _run(lib, x, tok, 8, scale=scale)
        assert int(r["status"].item()) == 0
        fine = [i for i in range(n) if float(x[i, int(tok[i])]) > low / 2]
        _check(r, x, tok, 8, dtype, scale=scale, rows=fine)
        for i in set(range(n)) - set(fine):
            assert r["logprob"][i].item() < -1e30


# two warps a row: the longest rows they take, whose chains are the longest of all
@pytest.mark.parametrize("dtype,V", [("bf16", 65536), ("f32", 32768), ("bf16", 30011)])
def test_narrow_rows(lib, dtype, V):
    n = 461
    assert _slices(n, V, dtype) == (1, 2)
    x = _logits(n, V, dtype, 1000)
    tok = _tokens(n, V)
    r = _run(lib, x, tok, 5)
    assert int(r["status"].item()) == 0
    _check(r, x, tok, 5, dtype, rows=[0, 1, 2, 230, 455, 456, 460])


@pytest.mark.parametrize("dtype,V", [("bf16", 70001), ("f32", 40001)])
@pytest.mark.parametrize("n", [20, 100, 200])
def test_slices_checked(lib, chk, n, dtype, V):  # noqa: F811
    # the bounds-checked build: no access out of range, and the same outputs
    x = _logits(n, V, dtype, 1100, stride=V + 3, offset=1)
    x[1, V // 2:] = -INF
    x[2] = 1.0
    tok = _tokens(n, V)
    a, b = (_run(m, x, tok, 32) for m in (lib, chk))
    assert int(b["status"].item()) == 0
    for k in ("logprob", "entropy", "lse", "idx", "top"):
        assert torch.equal(a[k], b[k]), k

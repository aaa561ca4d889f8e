"""ripple_token_logprobs against the oracle in 64 bits.

Tolerances, with d = scale (x - max) and S' the sum of exp(d) over all but the largest:
d is rounded twice (2^-23 relative); an exponential's relative error is 2^-22 and, for its
argument, 2^-23 |d| (terms of |d| > 17 count for less than their error allows); a sum of
V terms is built from chains of at most V / 256 + 64 additions, 2^-24 each:
e = 2^-22 + 2^-19 + (V / 256 + 64) 2^-24 relative to S', hence to log1p(S'), whose own
rounding is within. log P: 2^-22 |d| + e log1p(S'). Entropy log1p(S') + T / (1 + S'), T the
sum of exp(d) |d|: e of each term (T's terms carry 2^-23 more, within). lse adds 2^-23 of
|scale max|. Indices are equal."""
import numpy as np
import pytest
import torch

from oracle import ripple_oracle as O
from paper_2608_08684_gb300 import synth
from tests import paged_common as P

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _run(lib, logits, tokens=None, top=0, scale=0.0, entropy=True, lse=True, status=None):
    n = logits.shape[0]
    nan = lambda *s: torch.full(s, float("nan"), device=DEV)  # noqa: E731
    r = dict(entropy=nan(n) if entropy else None, lse=nan(n) if lse else None,
             logprob=nan(n) if tokens is not None else None,
             idx=torch.full((n, top), -9, dtype=torch.int32, device=DEV) if top else None,
             top=nan(n, top) if top else None,
             status=torch.zeros(1, dtype=torch.int32, device=DEV) if status is None else status)
    lib.ripple_token_logprobs(logits, tokens, r["logprob"], entropy_out=r["entropy"],
                              lse_out=r["lse"], top_idx=r["idx"], top_logprob=r["top"], scale=scale,
                              dev_status=r["status"])
    return r


def _check(r, logits, tokens=None, top=0, scale=1.0, rows=None):
    x = synth.to_f64(logits)
    V = x.shape[1]
    e = 2.0 ** -22 + 2.0 ** -19 + (V / 256 + 64) * 2.0 ** -24
    h = {k: None if t is None else t.cpu().numpy() for k, t in r.items()}
    for i in range(len(x)) if rows is None else rows:
        lp, ent = O.token_logprobs(x[i], scale)
        m = x[i].max()
        w = np.exp(scale * (x[i] - m))
        w[x[i].argmax()] = 0
        l1 = np.log1p(w.sum())
        d = np.where(np.isfinite(x[i]), scale * (x[i] - m), 0.0)
        T = (w * np.abs(d)).sum() / (1 + w.sum())

        def close(got, want, dist, what):
            if np.isinf(want):
                assert got == want, (what, i, got, want)
            else:
                # the oracle subtracts its log of the sum, of the size of the largest logit, from
                # the logit: its own last bit is larger than a log probability near 0
                assert abs(want - (dist - l1)) <= 2.0 ** -50 * (abs(scale * m) + abs(dist) + l1)
                want = dist - l1
                assert abs(got - want) <= 2.0 ** -22 * abs(dist) + e * l1 + 1e-30, (what, i, got, want)

        if h["entropy"] is not None:
            # as above: the oracle's -log p of the likeliest token has lost its last digits (and
            # sums of V terms, pairwise, carry up to log2 V + 8 roundings of 2^-53)
            assert abs(ent - (l1 + T)) <= 2.0 ** -46 * (abs(scale * m) + l1 + T)
            assert abs(h["entropy"][i] - (l1 + T)) <= 2 * e * (l1 + T) + 1e-30, (i, h["entropy"][i])
        if h["lse"] is not None:
            assert abs(h["lse"][i] - (scale * m + l1)) <= e * l1 + 2.0 ** -23 * (abs(scale * m) + l1), i
        if tokens is not None:
            t = int(tokens[i])
            if t < 0:
                assert h["logprob"][i] == 0
            else:
                close(h["logprob"][i], lp[t], d[t], "logprob")
        if top:
            want = O.top_tokens(x[i], top)
            assert h["idx"][i].tolist() == want.tolist(), (i, h["idx"][i], want)
            for j, t in enumerate(want):
                close(h["top"][i, j], lp[t], d[t], "top")


def _logits(n, V, dtype, seed, gain=2.5, peaks=4, stride=0, offset=0):
    """[n][V] logits with a few likely tokens, rows `stride` elements apart."""
    g = P.gen(seed)
    x = torch.randn((n, V), device=DEV, generator=g) * gain
    for _ in range(peaks):
        x[torch.arange(n, device=DEV), torch.randint(0, V, (n,), device=DEV, generator=g)] += 12
    x = x.to(P.DT[dtype])
    if stride:
        buf = torch.full((n * stride + offset + V,), float("nan"), dtype=x.dtype, device=DEV)
        view = buf[offset:].as_strided((n, V), (stride, 1))
        view.copy_(x)
        return view
    return x


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [1, 2, 7, 8, 9, 31, 33, 255, 1000, 4097, 32003, 128256])
@pytest.mark.parametrize("n", [1, 3, 41])
def test_vocabularies_and_rows(lib, n, V, dtype):
    x = _logits(n, V, dtype, 10 + V)
    tok = torch.randint(0, V, (n,), device=DEV, generator=P.gen(V)).to(torch.int32)
    top = min(V, 5)
    r = _run(lib, x, tok, top)
    assert int(r["status"].item()) == 0
    _check(r, x, tok, top, rows=[0, n // 2, n - 1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("stride,offset", [(5003, 0), (5003, 1), (5004, 3), (5008, 8), (6001, 5), (0, 0)])
def test_strides_and_alignments(lib, stride, offset, dtype):
    V = 5003
    x = _logits(6, V, dtype, 77, stride=stride or V, offset=offset)
    if stride == 0:  # one row for every token
        x = x[:1].expand(6, V)
    tok = P.i32([0, 1, V - 1, 2500, -1, 7])
    r = _run(lib, x, tok, 32, scale=0.7)
    assert int(r["status"].item()) == 0
    _check(r, x, tok, 32, scale=float(np.float32(0.7)))


@pytest.mark.parametrize("n", [1, 2, 5, 19, 20, 100, 153, 400, 700])
def test_row_counts(lib, n):
    # every way the rows may be spread over the GPU
    V = 9001
    x = _logits(n, V, "bf16", 500 + n)
    tok = torch.randint(0, V, (n,), device=DEV, generator=P.gen(n)).to(torch.int32)
    r = _run(lib, x, tok, 20)
    _check(r, x, tok, 20, rows=sorted({0, 1 % n, n // 2, n - 1}))
    again = _run(lib, x, tok, 20)
    for k in ("logprob", "entropy", "lse", "idx", "top"):
        assert torch.equal(r[k], again[k])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V,top", [(3, 1), (700, 32), (4097, 32), (30011, 5), (70001, 0)])
def test_more_rows_than_places(lib, V, top, dtype):
    n = 1999
    x = _logits(n, V, dtype, 600 + V)
    x[5::7] = 1.5                       # more ties than candidates
    x[6::7, : V // 2] = -float("inf")   # masked
    x[11::97, V // 3:] = -float("inf")
    tok = torch.randint(0, V, (n,), device=DEV, generator=P.gen(V)).to(torch.int32)
    r = _run(lib, x, tok, top, scale=1.25)
    assert int(r["status"].item()) == 0
    has = (x > -float("inf")).any(1)
    rows = [0, 5, 6, 455, 456, 1100, n - 1] + list(range(0, n, 61))
    _check(r, x, tok, top, scale=1.25, rows=[i for i in rows if bool(has[i])])
    again = _run(lib, x, tok, top, scale=1.25)
    few = _run(lib, x[800:1200], tok[800:1200], top, scale=1.25)  # split otherwise
    for k in ("logprob", "entropy", "lse", "idx", "top"):
        if r[k] is not None:
            a, b = r[k][has], again[k][has]
            assert torch.equal(a, b), k
            if k == "idx":
                assert torch.equal(r[k][800:1200][has[800:1200]], few[k][has[800:1200]])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("top", [1, 2, 31, 32])
def test_ties_go_to_the_lowest_index(lib, top, dtype):
    V = 20011
    g = P.gen(3)
    x = torch.randint(-3, 4, (6, V), device=DEV, generator=g).float()
    x[1] = 2.5                       # all equal
    x[2, 7000:] = 3                  # the largest ones side by side
    x[3] = 0.0
    x[3, ::3] = -0.0                 # 0 and -0 are equal
    x[4, :] = -1.0
    x[4, 19990:] = 4.0               # ties at the end
    x[5] = torch.arange(V, device=DEV) // 700  # ascending
    x = x.to(P.DT[dtype])
    r = _run(lib, x, P.i32([0] * 6), top)
    _check(r, x, P.i32([0] * 6), top)


@pytest.mark.parametrize("V,n", [(50000, 2), (50000, 300), (700, 5)])
def test_descending_and_clustered_rows(lib, V, n):
    # the largest logits next to one another, at either end, and spread by every small step
    x = torch.zeros(n, V, device=DEV)
    x[0] = -torch.arange(V, device=DEV).float() / 64
    x[1] = torch.arange(V, device=DEV).float() / 64
    for i in range(2, n):
        x[i, i % 97::(16 << (i % 9))] = 1.0 + torch.arange(len(x[i, i % 97::(16 << (i % 9))]), device=DEV) * 1e-3
    r = _run(lib, x, None, 32)
    _check(r, x, None, 32, rows=[i for i in (0, 1, 2, 3, 4, 9, 10, 150, 299) if i < n])


def test_masks(lib):
    V = 30000
    inf, low = float("inf"), torch.finfo(torch.float32).min
    x = _logits(9, V, "f32", 9)
    hide = torch.rand((9, V), device=DEV, generator=P.gen(4)) < 0.95
    x[0] = x[0].masked_fill(hide[0], -inf)
    x[1] = x[1].masked_fill(hide[1], low)
    x[2] = -inf
    x[2, 29999] = -3.0               # one token
    x[3] = -inf
    x[3, [5, 17000]] = torch.tensor([low, low], device=DEV)  # two of the lowest value
    x[4] = low                       # nothing but the lowest value
    x[5, :28000] = -inf
    x[6, 100:] = -inf
    x[7] = -inf
    x[7, :3] = torch.tensor([3e38, -3e38, 1e38], device=DEV)
    x[8] = 1e30
    tok = P.i32([1, 2, 29999, 17000, 7, 5, 50, 2, 11])
    r = _run(lib, x, tok, 32)
    assert int(r["status"].item()) == 0
    # rows whose differences overflow: by hand below
    _check(r, x, tok, 32, rows=[0, 1, 2, 3, 4, 5, 6, 8])
    assert r["logprob"][2].item() == 0 and r["entropy"][2].item() == 0
    assert r["entropy"][4].item() == pytest.approx(np.log(V), rel=1e-6)
    assert r["idx"][7].tolist() == [0, 2, 1] + list(range(3, 32))
    assert r["top"][7, 0].item() == 0 and r["entropy"][7].item() == 0
    assert (r["top"][7, 3:] == -inf).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_logits_of_every_size(lib, dtype):
    # masks of the lowest value beside infinite ones, logits and scales at the type's ends
    V = 4099
    low = torch.finfo(P.DT[dtype]).min
    g = P.gen(91)
    noise = torch.randn((2, V), device=DEV, generator=g)
    x = torch.full((3, V), low, dtype=P.DT[dtype], device=DEV)
    x[1, 77] = 0
    x[2, 100:] = low / 2
    x[:, ::3] = -float("inf")
    tok = P.i32([1, 77, 4000])
    r = _run(lib, x, tok, 4)
    assert int(r["status"].item()) == 0
    _check(r, x, tok, 4)
    for size, scale in ((1e36, 2e-36), (1e35, 2e-35), (1e-30, 1e30)):
        x = (noise * size).to(P.DT[dtype])
        x[:, 5::3] = -float("inf")
        tok = P.i32([0, 3])
        r = _run(lib, x, tok, 4, scale=scale)
        _check(r, x, tok, 4, scale=float(np.float32(scale)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_without_a_distribution(lib, dtype):
    V = 5000
    x = _logits(5, V, dtype, 21)
    clean = x.clone()
    x[1] = -float("inf")
    x[2, 4321] = float("nan")
    x[3, 77] = float("inf")
    tok = P.i32([3, 3, 3, 3, 3])
    r = _run(lib, x, tok, 5)
    assert int(r["status"].item()) == 0
    _check(r, clean, tok, 5, rows=[0, 4])
    for i in (1, 2, 3):
        assert torch.isnan(r["logprob"][i]) and torch.isnan(r["entropy"][i]), i
        assert torch.isnan(r["top"][i]).all(), i
        assert ((r["idx"][i] >= 0) & (r["idx"][i] < V)).all() and len(set(r["idx"][i].tolist())) == 5
    assert r["lse"][1].item() == -float("inf") and torch.isnan(r["lse"][2:4]).all()


def test_precision_near_certainty(lib):
    # one token of probability nearly 1: its log probability and the entropy are small numbers
    # with all their digits
    V = 128256
    x = torch.randn((4, V), device=DEV, generator=P.gen(31))
    for i, gap in enumerate((18.0, 25.0, 40.0, 80.0)):
        x[i, 1000 * i] = gap
    tok = P.i32([0, 1000, 2000, 3000])
    r = _run(lib, x, tok, 1)
    _check(r, x, tok, 1)
    assert -1e-2 < r["logprob"][0].item() < 0 and -1e-12 < r["logprob"][2].item() < 0


def test_padding_and_tokens_outside(lib):
    V = 100
    x = _logits(4, V, "f32", 41)
    r = _run(lib, x, P.i32([-1, 5, -100, 99]))
    assert int(r["status"].item()) == 0
    _check(r, x, P.i32([-1, 5, -100, 99]))
    r = _run(lib, x, P.i32([0, 100, 3, 2 ** 31 - 1]))
    assert int(r["status"].item()) == lib.EBOUNDS
    assert torch.isnan(r["logprob"]).tolist() == [False, True, False, True]
    _check(r, x, None)


def test_each_output_alone(lib):
    x = _logits(3, 4000, "bf16", 51)
    tok = P.i32([1, 2, 3])
    _check(_run(lib, x, tok, entropy=False, lse=False), x, tok)
    _check(_run(lib, x, None, lse=False), x)
    _check(_run(lib, x, None, entropy=False), x)
    _check(_run(lib, x, None, 3, entropy=False, lse=False), x, None, 3)
    idx = torch.zeros(3, 7, dtype=torch.int32, device=DEV)
    lib.ripple_token_logprobs(x, top_idx=idx)  # indices without their log probabilities
    torch.cuda.synchronize()
    assert idx[1].tolist() == O.top_tokens(synth.to_f64(x[1]), 7).tolist()
    before = lib.ripple_kernel_launches()
    _run(lib, x[:0], tok[:0], 3)
    assert lib.ripple_kernel_launches() == before


def test_rows_far_apart(lib):
    # row offsets beyond 2^31 elements
    V, stride = 1000, (1 << 30) + 24
    buf = torch.empty(2 * stride + V, dtype=torch.bfloat16, device=DEV)
    x = buf.as_strided((3, V), (stride, 1))
    x.copy_(_logits(3, V, "bf16", 61))
    tok = P.i32([1, 2, 999])
    _check(_run(lib, x, tok, 5), x, tok, 5)


def test_graph_and_stream(lib):
    x = _logits(7, 50001, "bf16", 71)
    tok = P.i32(list(range(7)))
    want = _run(lib, x, tok, 9)
    torch.cuda.synchronize()
    out = [torch.zeros(7, device=DEV) for _ in range(3)]
    idx, lp = torch.zeros(7, 9, dtype=torch.int32, device=DEV), torch.zeros(7, 9, device=DEV)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        with torch.cuda.graph(g, stream=s):
            lib.ripple_token_logprobs(x, tok, out[0], out[1], out[2], idx, lp)
        for _ in range(3):
            g.replay()
    s.synchronize()
    for a, k in zip(out + [idx, lp], ("logprob", "entropy", "lse", "idx", "top")):
        assert torch.equal(a, want[k])

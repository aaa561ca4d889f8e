"""Shared pieces of the tests of scores and scales far from one another over 8-bit pages."""
import numpy as np
import torch

from tests import paged8_common as P8
from tests import paged_common as P

DEV = "cuda"
LN2, LOG2E = float(np.log(2.0)), float(np.log2(np.e))


def codes(x):
    return torch.as_tensor(x, device=DEV).float().to(torch.float8_e4m3fn).view(torch.uint8)


def rows(pool, b, n):
    at = [pool.place(b, r) for r in range(n)]
    return [torch.tensor(x, device=DEV) for x in zip(*at)]


def far_pool(lib, lens, d, dtype, seed, width):
    """Keys of about -1 in every dim, the later ones smaller in magnitude."""
    pool = P8.Pool8(lib, lens, 1, d, 16, dtype, seed, spread=0.5, width=width)
    rng = np.random.default_rng(seed)
    for b, n in enumerate(lens):
        if n == 0:
            continue
        size = np.linspace(1.9, 1.1, n)[:, None] * (1 + 0.06 * rng.standard_normal((n, d)))
        p, s = rows(pool, b, n)
        pool.k[p, 0, s] = codes(-size)
        pool.ks[p, 0, s] = 127
    return pool


def far_queries(shape, dtype, seed):
    return (1 + 0.1 * P.randn(shape, "f32", seed)).to(P.DT[dtype])


def one_hot(q, k, v, scale):
    """(the rows of q whose best key is clear of the next, as far as fp32 scores tell them apart; that
    key's value, which has all the weight)"""
    x = q.double().cpu().numpy() @ k.T * scale
    two = np.sort(x, axis=1)[:, -2:]
    clear = two[:, 1] - two[:, 0] > 64 * 2.0 ** -21 * np.abs(x).max(1) + 40
    assert clear.sum() > len(x) // 2
    return clear, v[x.argmax(1)][clear]


def bound(kind, x, size, want):
    """What an output may be off by. A score x (log2 units) is an fp32 sum of products that matrix
    instructions cut off, times a rounded scale: off by 2^-21 |x| at most; two rows' weights are
    then off by 2^-20 |x| ln 2 against each other, an output by that times the values' size, sum(p |v|),
    and once more by the sum's share. Beside that the decode's 1e-4 of that size; outputs in bf16 are
    rounded (2^-8 of themselves) and come from probabilities in fp16 (2^-11 of the size)."""
    rel = 2 * 2.0 ** -20 * np.abs(x) * LN2 + 1e-4
    if kind == "q8-bf16":
        return (rel + 2.0 ** -11) * size + 2.0 ** -8 * np.abs(want)
    return rel * size

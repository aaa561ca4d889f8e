"""Helpers of the paged-cache tests: pools with their pages handed out at random, in the
layouts a program may have, and the reference in 64 bits."""
from __future__ import annotations

import numpy as np
import torch

from oracle import ripple_oracle as O
from paper_2608_08684_gb300 import synth

DEV = "cuda"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}  # of a rounding, relative


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def randn(shape, dtype, seed):
    return torch.randn(shape, dtype=DT[dtype], device=DEV, generator=gen(seed))


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


class Pool:
    """Pools of pages for rows[b] rows of every sequence, and the block table, entries
    behind a sequence's last page invalid. layout: "heads" [page][head][row][d], "rows"
    [page][row][head][d], "pair" [page][k, v][head][row][d] (one allocation)."""

    def __init__(self, lib, rows, heads, d, page, dtype, seed, layout="heads", fill=None, width=0):
        need = [-(-n // page) for n in rows]
        self.n_pages = max(1, sum(need)) + 2
        width = max(width, max(need), 1)
        rng = np.random.default_rng(seed)
        ids = rng.permutation(self.n_pages)
        table = np.full((len(rows), width), -7, np.int32)
        at = 0
        for b, n in enumerate(need):
            table[b, :n] = ids[at:at + n]
            at += n
        self.spare = ids[at:].tolist()  # pages of no sequence
        n = self.n_pages
        if layout == "heads":
            k, v = (randn((n, heads, page, d), dtype, seed + i) for i in (1, 2))
        elif layout == "rows":
            k, v = (randn((n, page, heads, d), dtype, seed + i).transpose(1, 2) for i in (1, 2))
        else:
            both = randn((n, 2, heads, page, d), dtype, seed + 1)
            k, v = both[:, 0], both[:, 1]
        if fill is not None:
            k.fill_(fill)
            v.fill_(fill)
        self.k, self.v, self.page, self.heads, self.d = k, v, page, heads, d
        self.np_table = table
        self.table = torch.from_numpy(table).to(DEV)
        self.cache = lib.PagedCache(k, v, self.table)
        self.rows = list(rows)

    def seq(self, which, b, n=None):
        """The first n rows of sequence b as float64 [heads][n][d]."""
        n = self.rows[b] if n is None else n
        t = {"k": self.k, "v": self.v}[which]
        pages = torch.from_numpy(self.np_table[b, :-(-n // self.page)].astype(np.int64)).to(DEV)
        x = t[pages].transpose(0, 1).reshape(self.heads, -1, self.d)[:, :n]
        return synth.to_f64(x)

    def place(self, b, r):
        return int(self.np_table[b, r // self.page]), r % self.page


def run_decode(lib, pool, q, lens, scale=0.0, lse=True, ws=None, status=None):
    B, Hq, d = q.shape
    need = lib.ripple_paged_decode_workspace_bytes(pool.cache, Hq)
    ws = torch.randint(0, 256, (need,), dtype=torch.uint8, device=DEV) if ws is None else ws
    out = torch.full((B, Hq, d), float("nan"), device=DEV)
    ls = torch.full((B, Hq), float("nan"), device=DEV) if lse else None
    status = torch.zeros(1, dtype=torch.int32, device=DEV) if status is None else status
    lib.ripple_paged_decode_attn(pool.cache, q, lens, out, ws, lse=ls, scale=scale,
                                 dev_status=status)
    return out, ls, status


def decode_ref(pool, q, lens, scale=None):
    """(out [B][Hq][d], lse [B][Hq]) in 64 bits."""
    B, Hq, d = q.shape
    G = Hq // pool.heads
    scale = d ** -0.5 if scale is None else scale
    out, lse = np.zeros((B, Hq, d)), np.full((B, Hq), -np.inf)
    for b, n in enumerate(lens):
        if n <= 0:
            continue
        k, v = pool.seq("k", b, n), pool.seq("v", b, n)
        for h in range(pool.heads):
            qq = synth.to_f64(q[b, h * G:(h + 1) * G])
            out[b, h * G:(h + 1) * G] = O.decode_attention(qq, k[h], v[h], scale)
            lse[b, h * G:(h + 1) * G] = O.attention_lse(qq, k[h], scale)
    return out, lse

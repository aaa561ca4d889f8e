"""Shared pieces of the tests of 8-bit paged caches and of drafted tokens: pools with tables,
references in 64 bits."""
import numpy as np
import torch

from tests import paged_common as P

DEV = "cuda"


def quantise64(x):
    """Rows of a float64 array [..][d] as (codes' values, scale bytes), from the definition: the
    least e >= -120 with max |x| <= 448 2^e, x 2^-e to the nearest e4m3 value, even at ties (at
    most 240 where e is 120); byte 255 and zeros for a row that is not finite."""
    x = np.asarray(x, np.float64)
    with np.errstate(all="ignore"):
        a = np.abs(x).max(-1)
        finite = np.isfinite(a)
        m, ex = np.frexp(np.where(finite, a, 1.0))  # m in [1/2, 1)
        e = np.maximum(np.where(a == 0, -120, ex - 9 + (m > 0.875)), -120)
        y = np.where(finite[..., None], x, 0.0) * np.exp2(-e.astype(np.float64))[..., None]
        step = np.exp2(np.floor(np.log2(np.maximum(np.abs(y), 2.0 ** -6))) - 3)
        c = np.round(y / step) * step  # numpy rounds half to even
    c = np.where((e == 120)[..., None], np.clip(c, -240, 240), c)
    return c, np.where(finite, e + 127, 255).astype(np.uint8)


def scale64(byte):
    return np.where(byte == 255, np.nan, np.exp2(byte.astype(np.float64) - 127))


class Pool8:
    """P.Pool in 8 bits: pools of codes with scales, filled with quantised normal rows whose
    sizes differ by powers of ten. gap: bytes between a row's codes and the next row's."""

    def __init__(self, lib, rows, heads, d, page, dtype, seed, layout="heads", gap=0, spread=1.0,
                 fill=True, width=0):
        need = [-(-n // page) for n in rows]
        self.n_pages = n = max(1, sum(need)) + 2
        width = max(width, max(need), 1)
        rng = np.random.default_rng(seed)
        ids = rng.permutation(n)
        table = np.full((len(rows), width), -7, np.int32)
        at = 0
        for b, k in enumerate(need):
            table[b, :k] = ids[at:at + k]
            at += k
        self.spare = ids[at:].tolist()
        lead = (n, heads, page) if layout == "heads" else (n, page, heads)

        def pool(i):
            x = torch.randn(lead + (d,), dtype=torch.float64, device=DEV, generator=P.gen(seed + i))
            size = torch.randn(lead, dtype=torch.float64, device=DEV, generator=P.gen(seed + 7 + i))
            x = x * torch.exp2(spread * size)[..., None]
            a = x.abs().amax(-1)
            e = torch.ceil(torch.log2(a / 448)).clamp(-120, 120)
            codes = (x / torch.exp2(e)[..., None]).clamp(-448, 448).float().to(torch.float8_e4m3fn)
            held = torch.zeros(lead + (d + gap,), dtype=torch.uint8, device=DEV)[..., :d]
            s = torch.full(lead, 127, dtype=torch.uint8, device=DEV)
            if fill:
                held.copy_(codes.view(torch.uint8))
                s.copy_((e + 127).to(torch.uint8))
            if layout == "rows":
                held, s = held.transpose(1, 2), s.transpose(1, 2)
            return held, s

        self.k, self.ks = pool(1)
        self.v, self.vs = pool(2)
        self.page, self.heads, self.d, self.rows = page, heads, d, list(rows)
        self.np_table = table
        self.dtype = P.DT[dtype]
        self.table = torch.from_numpy(table).to(DEV)
        self.lib = lib
        self.bind()

    def bind(self):
        f8, e8 = torch.float8_e4m3fn, torch.float8_e8m0fnu
        self.cache = self.lib.PagedCache(self.k.view(f8), self.v.view(f8), self.table,
                                         k_scales=self.ks.view(e8), v_scales=self.vs.view(e8),
                                         dtype=self.dtype)

    def values(self, which, pages=slice(None)):
        """[pages][heads][rows][d] in 64 bits."""
        codes, s = {"k": (self.k, self.ks), "v": (self.v, self.vs)}[which]
        x = codes[pages].contiguous().view(torch.float8_e4m3fn).double().cpu().numpy()
        return x * scale64(s[pages].cpu().numpy())[..., None]

    def seq(self, which, b, n=None):
        n = self.rows[b] if n is None else n
        pages = torch.from_numpy(self.np_table[b, :-(-n // self.page)].astype(np.int64)).to(DEV)
        x = self.values(which, pages)
        return x.transpose(1, 0, 2, 3).reshape(self.heads, -1, self.d)[:, :n]

    def place(self, b, r):
        return int(self.np_table[b, r // self.page]), r % self.page


def any_pool(lib, kind, rows, heads, d, page, seed, layout="heads", width=0):
    """kind: bf16, f32, or the queries' type over 8-bit pages: q8-bf16, q8-f32."""
    if kind.startswith("q8"):
        return Pool8(lib, rows, heads, d, page, kind[3:], seed, layout, width=width)
    return P.Pool(lib, rows, heads, d, page, kind, seed, layout, width=width)


def type_of(kind):
    return kind[3:] if kind.startswith("q8") else kind


def random_masks(counts, seed):
    """Bits of random trees for sequences of counts tokens."""
    rng = np.random.default_rng(seed)
    out = []
    for n in counts:
        mine = []
        for j in range(n):
            parent = int(rng.integers(0, j)) if j else -1
            mine.append((mine[parent] if parent >= 0 else 0) | 1 << j)
        out += mine
    return out


def to_i64(masks):
    return torch.tensor([m - (1 << 64) if m >> 63 else m for m in masks], dtype=torch.int64, device=DEV)


def run_tree(lib, pool, q, lens, masks=None, starts=None, max_tokens=None, scale=0.0, ws=None,
             status=None, lse=True):
    most = max_tokens or (q.shape[1] if starts is None else 64)
    need = lib.ripple_paged_tree_workspace_bytes(pool.cache, q.shape[-2], most)
    ws = torch.randint(0, 256, (need,), dtype=torch.uint8, device=DEV) if ws is None else ws
    out = torch.full(q.shape, float("nan"), dtype=q.dtype, device=DEV)
    ls = torch.full(q.shape[:-1], float("nan"), device=DEV) if lse else None
    status = torch.zeros(1, dtype=torch.int32, device=DEV) if status is None else status
    lib.ripple_paged_tree_attn(pool.cache, q, lens, out, ws, masks=masks, seq_starts=starts,
                               max_tokens=max_tokens, lse=ls, scale=scale, dev_status=status)
    return out, ls, status


def tree_ref(pool, q, lens, counts, masks, scale=None, missing=()):
    """q [tokens][Hq][d] (sequence after sequence); (out, lse, sum of p |v|) in 64 bits. missing:
    (sequence, row) that are left out. Values of hidden rows are not touched."""
    T, Hq, d = q.shape
    H, G = pool.heads, Hq // pool.heads
    scale = d ** -0.5 if scale is None else scale
    qq = q.double().cpu().numpy()
    out, size = np.zeros((T, Hq, d)), np.zeros((T, Hq, d))
    lse = np.full((T, Hq), -np.inf)
    t0 = 0
    for b, (n, m) in enumerate(zip(lens, counts)):
        if n > 0:
            k, v = pool.seq("k", b, n), pool.seq("v", b, n)
            for i in range(m):
                bits = (1 << (i + 1)) - 1 if masks is None else masks[t0 + i]
                rows = [r for r in range(max(0, n - m), n) if bits >> (r - (n - m)) & 1]
                rows = list(range(max(0, n - m))) + rows
                rows = np.array([r for r in rows if (b, r) not in missing], int)
                if len(rows) == 0:
                    continue
                for h in range(H):
                    hs = slice(h * G, (h + 1) * G)
                    with np.errstate(all="ignore"):
                        x = qq[t0 + i, hs] @ k[h][rows].T * scale
                        top = x.max(1, keepdims=True)
                        top = np.where(np.isfinite(top), top, 0.0)
                        p = np.exp(x - top)
                        s = p.sum(1, keepdims=True)
                        lse[t0 + i, hs] = (top + np.log(s))[:, 0]
                        p = p / np.where(s > 0, s, 1.0)
                        out[t0 + i, hs] = p @ v[h][rows]
                        size[t0 + i, hs] = p @ np.abs(v[h][rows])
        t0 += m
    return out, lse, size

"""Operators of a serving program whose paged KV cache is held in 8 bits, or which has several
drafted tokens of a sequence looked at in one step, as such a program calls them.

  append8  new tokens' keys and values into a paged cache of 8-bit codes with a scale a row and
           head, rotated on the way, with the queries rotated in the same pass
  decode8  attention of one new token per sequence over such a cache
  tree     attention of a tree of drafted tokens per sequence over a paged cache (bf16, fp32
           or 8 bits): every token sees the rows before the draft and those drafted tokens
           that its mask names
  keep     the accepted drafted tokens' rows moved up behind the rows before the draft, in
           every layer, and the new lengths

With `own` false the operators are computed in their plain form: elementary torch
operations in 32 bits (angles in 64), rounded once at the end. `exact` computes the
same from the definitions in 64 bits, one sequence at a time.

A row x of d values is held as codes c_i (e4m3) and a scale 2^e: e is the least whole number
with max |x_i| <= 448 2^e, and c_i is x_i 2^-e rounded to the nearest e4m3 value (even ones
at ties).

Shapes are those of the repository's synthetic workloads (8B: 32 query and 8 KV heads
of 128 dims; 70B: 64 and 8; caches of a few hundred rows after compression up to 128k
uncompressed ones) and of odd sizes between them. Keys are N(0, 1) with a per-channel
lognormal(0, 0.5) scale, values N(0, 1), queries N(0, 1) with a gain of 2 (attention as peaked
as a trained model's).
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda"
_DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # a decode step of a batch padded for a captured graph (8 sequences idle)
        dict(name="append8_batch", kind="append8", dtype="bf16", q_heads=32, kv_heads=8, dim=128,
             page=16, rot=128, inter=False, batch=72, new_lo=1, new_hi=1, old_lo=1, old_hi=32767,
             idle=8, ragged=False, layout="heads", mix=1),
        # whole prompts
        dict(name="append8_prompts", kind="append8", dtype="bf16", q_heads=32, kv_heads=8, dim=128,
             page=64, rot=128, inter=False, batch=6, new_lo=4000, new_hi=16384, old_lo=1,
             old_hi=300, idle=0, ragged=True, layout="heads", mix=2),
        # one sequence over a compressed cache
        dict(name="decode8_short", kind="decode8", dtype="bf16", q_heads=32, kv_heads=8, dim=128,
             page=16, batch=1, lo=470, hi=470, layout="heads", mix=3),
        # continuous batching: 64 sequences, from an idle one to 32k tokens
        dict(name="decode8_ragged", kind="decode8", dtype="bf16", q_heads=32, kv_heads=8, dim=128,
             page=16, batch=64, lo=64, hi=32768, layout="heads", mix=4),
        # fp32 queries, seven of them a KV head, the heads of a row side by side
        dict(name="decode8_f32_g7", kind="decode8", dtype="f32", q_heads=28, kv_heads=4, dim=64,
             page=32, batch=9, lo=1000, hi=60000, layout="rows", mix=5),
        # one sequence, a chain of four drafted tokens over a compressed cache
        dict(name="tree_chain", kind="tree", dtype="bf16", bits=16, q_heads=32, kv_heads=8, dim=128,
             page=16, batch=1, new_lo=4, new_hi=4, lo=900, hi=900, chain=True, ragged=False,
             layout="heads", mix=6),
        # continuous batching with a tree of 2 to 12 tokens for every sequence
        dict(name="tree_batch", kind="tree", dtype="bf16", bits=16, q_heads=32, kv_heads=8, dim=128,
             page=32, batch=48, new_lo=2, new_hi=12, lo=64, hi=32768, chain=False, ragged=True,
             layout="heads", mix=7),
        # large trees over long caches, eight query heads a KV head
        dict(name="tree_long_g8", kind="tree", dtype="bf16", bits=16, q_heads=64, kv_heads=8,
             dim=128, page=64, batch=3, new_lo=64, new_hi=64, lo=30000, hi=32768, chain=False,
             ragged=False, layout="heads", mix=8),
        # the batch over a cache in 8 bits
        dict(name="tree8_batch", kind="tree", dtype="bf16", bits=8, q_heads=32, kv_heads=8, dim=128,
             page=16, batch=32, new_lo=16, new_hi=16, lo=500, hi=32768, chain=False, ragged=False,
             layout="heads", mix=9),
        # fp32, seven query heads a KV head, a ragged batch, the heads of a row side by side
        dict(name="tree_f32_g7", kind="tree", dtype="f32", bits=32, q_heads=28, kv_heads=4, dim=64,
             page=32, batch=7, new_lo=1, new_hi=9, lo=100, hi=6000, chain=False, ragged=True,
             layout="rows", mix=10),
        # one sequence, all layers
        dict(name="keep_one", kind="keep", dtype="bf16", bits=16, layers=32, kv_heads=8, dim=128,
             page=16, batch=1, new=16, kept=4, lo=900, hi=900, layout="heads", mix=11),
        # a batch, all layers, in 8 bits
        dict(name="keep8_batch", kind="keep", dtype="bf16", bits=8, layers=32, kv_heads=8, dim=128,
             page=16, batch=64, new=16, kept=4, lo=20, hi=300, layout="heads", mix=12),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


# (query heads, KV heads, head dim)
_HEADS = [(32, 8, 128), (32, 8, 128), (64, 8, 128), (28, 4, 128), (8, 8, 64), (40, 4, 64),
          (5, 1, 128), (16, 1, 64)]


def draw(rng):
    kind = rng.choice(["append8", "decode8", "decode8", "tree", "tree", "tree", "keep"])
    hq, hkv, dim = rng.choice(_HEADS)
    c = dict(kind=kind, dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]), kv_heads=hkv, dim=dim,
             page=rng.choice([1, 8, 16, 16, 32, 64, 128, 256]),
             layout=rng.choice(["heads", "heads", "rows"]), mix=rng.randrange(1, 1 << 30))
    if kind != "keep":
        c["q_heads"] = hq
    if kind in ("tree", "keep"):
        c["bits"] = rng.choice([8, 32 if c["dtype"] == "f32" else 16])
    if kind == "keep":
        c["layers"] = rng.choice([1, 8, 32, 80])
        c["new"] = _log(rng, 2, 64)
        c["kept"] = rng.randrange(0, min(12, c["new"]))
        c["batch"] = _log(rng, 1, max(1, 2048 // c["layers"]))
        c["hi"] = _log(rng, 8, max(16, 600_000 // (c["layers"] * c["batch"])))
        c["lo"] = _log(rng, 1, c["hi"])
        return c
    if kind == "append8":
        c["rot"] = rng.choice([dim, dim, dim, dim // 2])
        c["inter"] = rng.choice([False, False, True])
        c["ragged"] = rng.choice([False, True])
        if c["ragged"]:
            c["batch"] = _log(rng, 1, 16)
            most = 44_000 * 6144 // ((hq + 2 * hkv) * dim * (2 if c["dtype"] == "f32" else 1))
            c["new_hi"] = _log(rng, 16, min(16384, most // c["batch"]))
            c["new_lo"] = _log(rng, 1, c["new_hi"])
        else:
            c["batch"] = _log(rng, 1, 256)
            c["new_lo"] = c["new_hi"] = rng.choice([1, 1, 1, 4])
        c["old_lo"], c["old_hi"] = 1, _log(rng, 16, 131072 // max(1, c["batch"] // 16))
        c["idle"] = 0 if c["ragged"] or c["batch"] < 4 else rng.choice([0, c["batch"] // 8])
        return c
    # at most about the bytes and operations of the largest listed steps, also if every sequence
    # were the longest
    e = 1 if kind == "decode8" else c["bits"] // 8
    if kind == "tree":
        c["ragged"] = rng.choice([False, True])
        c["chain"] = rng.choice([False, False, True])
        c["new_hi"] = _log(rng, 1, 64)
        c["new_lo"] = _log(rng, 1, c["new_hi"]) if c["ragged"] else c["new_hi"]
    c["batch"] = _log(rng, 1, 128 if kind == "tree" else 256)
    most = min(131072, 1_000_000_000 // (2 * e * hkv * dim * c["batch"]))
    if kind == "tree":
        most = min(most, 150_000_000_000 // (4 * c["batch"] * c["new_hi"] * hq * dim))
        if c["dtype"] == "f32":  # without tensor cores
            most = min(most, 10_000_000_000 // (4 * c["batch"] * c["new_hi"] * hq * dim))
    c["hi"] = _log(rng, 16, max(64, most))
    c["lo"] = _log(rng, 1, c["hi"])
    return c


# ------------------------------------------------------------------ inputs


def _gen(seed, tag):
    g = torch.Generator(device=DEV)
    g.manual_seed((int(seed) * 1000003 + tag) & ((1 << 62) - 1))
    return g


def _randn(shape, dtype, seed, tag):
    return torch.randn(shape, dtype=dtype, device=DEV, generator=_gen(seed, tag))


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _lens(case):
    """(new tokens, rows once they are in) of every sequence; the same for every seed up to
    their order. A decode batch of eight or more has an empty sequence and one of one row, a
    tree's batch an idle sequence and one with nothing before the draft."""
    c, rng = case, random.Random(case["mix"])
    B = c["batch"]
    if c["kind"] == "decode8":
        rows = [_log(rng, c["lo"], c["hi"]) for _ in range(B)]
        if B >= 8:
            rows[:2] = [0, 1]
        return [1] * B, rows
    if c["kind"] == "keep":
        return [c["new"]] * B, [c["new"] + _log(rng, c["lo"], c["hi"]) for _ in range(B)]
    new = [_log(rng, c["new_lo"], c["new_hi"]) for _ in range(B)]
    if c["kind"] == "tree":
        rows = [n + _log(rng, c["lo"], c["hi"]) for n in new]
        if B >= 8:
            rows[:2] = [0, new[1]]
        return new, rows
    rows = [n + _log(rng, c["old_lo"], c["old_hi"]) for n in new]
    for b in range(c["idle"]):
        rows[B - 1 - b] = 0
    return new, rows


def _pow2(scales):
    """2^(s - 127) of bytes s in 1..254."""
    return (scales.to(torch.int32) << 23).view(torch.float32)


def _quantise(x):
    """Rows (the last dim) as e4m3 codes and scale bytes; bytes both."""
    x = x.float()
    mantissa, exponent = torch.frexp(x.abs().amax(-1))  # mantissa in [1/2, 1)
    e = exponent - 9 + (mantissa > 0.875).int()  # 448 = 0.875 2^9
    e = torch.where(mantissa == 0, -120, e).clamp(-120, 120)
    codes = (x * _pow2(127 - e)[..., None]).to(torch.float8_e4m3fn)
    return codes.view(torch.uint8), (e + 127).to(torch.uint8)


def _table(c, seed, rows):
    """Pages for `rows` rows of every sequence, handed out in random order: their number and the
    table. Entries behind a sequence's last page are no pages."""
    need = [max(1, -(-n // c["page"])) for n in rows]
    n_pages, width = sum(need), max(need)
    perm = torch.randperm(n_pages, device=DEV, generator=_gen(seed, 20)).to(torch.int32)
    starts = [0]
    for n in need:
        starts.append(starts[-1] + n)
    at = _i32(starts[:-1])[:, None] + torch.arange(width, device=DEV)[None]
    table = perm[at.clamp(max=n_pages - 1)]
    table = torch.where(torch.arange(width, device=DEV)[None] < _i32(need)[:, None], table, -1)
    return n_pages, table.contiguous()


def _pools(c, seed, rows, fill, bits):
    """The pools of one layer and the table: k, v (and k_scales, v_scales), 8-bit ones as bytes."""
    ps, H, D, dt = c["page"], c["kv_heads"], c["dim"], _DT[c["dtype"]]
    n_pages, table = _table(c, seed, rows)
    # heads: [page][head][row][dim]; rows: [page][row][head][dim]
    shape = (n_pages, H, ps, D) if c["layout"] == "heads" else (n_pages, ps, H, D)
    out = {}
    for tag, name in enumerate(("k", "v")):
        if not fill:
            x = torch.zeros(shape, dtype=torch.uint8 if bits == 8 else dt, device=DEV)
            s = torch.full(shape[:3], 127, dtype=torch.uint8, device=DEV)
        else:
            x = _randn(shape, dt, seed, 22 + tag)
            if name == "k":
                scale = torch.exp(0.5 * _randn((H, D), torch.float32, seed, 21)).to(dt)
                x.mul_(scale[:, None] if c["layout"] == "heads" else scale)
            if bits == 8:
                x, s = _quantise(x)
        out[name] = x.transpose(1, 2) if c["layout"] == "rows" else x
        if bits == 8:
            out[name + "_scales"] = s.transpose(1, 2) if c["layout"] == "rows" else s
    return out, table


def _held(bits, pools):
    """The pools as a program holds them: 8-bit ones with the types of their values."""
    if bits != 8:
        return pools
    return {n: x.view(torch.float8_e8m0fnu if n.endswith("_scales") else torch.float8_e4m3fn)
            for n, x in pools.items()}


def _inv_freq(c):
    """Base 500000, the usual spacing."""
    return [500000.0 ** (-2.0 * j / c["rot"]) for j in range(c["rot"] // 2)]


def _starts(new):
    starts = [0]
    for m in new:
        starts.append(starts[-1] + m)
    return starts


def _shuffled(seed, *lists):
    order = list(range(len(lists[0])))
    random.Random(seed).shuffle(order)
    return [[x[i] for i in order] for x in lists]


def _prepare_append8(c, seed):
    new, rows = _shuffled(seed, *_lens(c))
    B, Hq, H, D, dt = c["batch"], c["q_heads"], c["kv_heads"], c["dim"], _DT[c["dtype"]]
    pools, table = _pools(c, seed, rows, False, 8)
    n = sum(new)
    room = n + 13 if c["ragged"] else n  # a ragged batch's buffers are longer than its tokens
    # the fused projection's output, q, k and v side by side in a token's row
    qkv = _randn((room, Hq + 2 * H, D), dt, seed, 2)
    q_out = torch.zeros((room, Hq, D), dtype=dt, device=DEV)
    if not c["ragged"]:
        qkv = qkv.view(B, new[0], Hq + 2 * H, D)
        q_out = q_out.view(B, new[0], Hq, D)
    q, k, v = qkv.split([Hq, H, H], dim=-2)
    # a compressed cache's rows are fewer than the positions behind it
    first = [r - m + (r // 2) for r, m in zip(rows, new)]
    pos = torch.cat([torch.arange(m, device=DEV) + f for f, m in zip(first, new)])
    pos = torch.cat([pos, torch.zeros(room - n, dtype=pos.dtype, device=DEV)]).to(torch.int32)
    return dict(kind="append8", n=n, B=B, page=c["page"], rot=c["rot"], inter=c["inter"],
                inv_freq=_inv_freq(c), q=q, k=k, v=v, q_out=q_out, pos=pos.view(q.shape[:-2]),
                starts=_i32(_starts(new)) if c["ragged"] else None, lens=_i32(rows), pools=pools,
                table=table)


def _prepare_decode8(c, seed):
    (rows,) = _shuffled(seed, _lens(c)[1])
    B, Hq, D, dt = c["batch"], c["q_heads"], c["dim"], _DT[c["dtype"]]
    pools, table = _pools(c, seed, rows, True, 8)
    return dict(kind="decode8", bits=8, most=max(rows), page=c["page"], lens=_i32(rows), pools=pools,
                table=table, q=_randn((B, Hq, D), dt, seed, 3).mul_(2),
                out=torch.zeros((B, Hq, D), device=DEV), lse=torch.zeros((B, Hq), device=DEV))


def _trees(new, seed):
    """Masks of random trees: every token sees its parent's tokens and itself."""
    rng = random.Random(seed)
    masks = []
    for n in new:
        own_masks = []
        for j in range(n):
            parent = rng.randrange((j - 1) // 3, j) if j else -1
            m = (own_masks[parent] if parent >= 0 else 0) | 1 << j
            own_masks.append(m)
        masks += own_masks
    return torch.tensor([m - (1 << 64) if m >> 63 else m for m in masks], dtype=torch.int64,
                        device=DEV)


def _prepare_tree(c, seed):
    new, rows = _shuffled(seed, *_lens(c))
    B, Hq, D, dt = c["batch"], c["q_heads"], c["dim"], _DT[c["dtype"]]
    pools, table = _pools(c, seed, rows, True, c["bits"])
    n = sum(new)
    room = n + 5 if c["ragged"] else n
    lead = (room,) if c["ragged"] else (B, new[0])
    masks = None
    if not c["chain"]:
        masks = torch.zeros(room, dtype=torch.int64, device=DEV)
        masks[:n] = _trees(new, seed)
        masks = masks.view(lead)
    return dict(kind="tree", bits=c["bits"], n=n, B=B, most=max(rows), most_new=max(new),
                page=c["page"], lens=_i32(rows), starts=_i32(_starts(new)) if c["ragged"] else None,
                pools=pools, table=table, masks=masks,
                q=_randn(lead + (Hq, D), dt, seed, 3).mul_(2),
                out=torch.zeros(lead + (Hq, D), dtype=dt, device=DEV),
                lse=torch.zeros(lead + (Hq,), device=DEV))


def _prepare_keep(c, seed):
    new, rows = _lens(c)
    L, B = c["layers"], c["batch"]
    per_layer = [_pools(c, seed + l, rows, True, c["bits"]) for l in range(L)]
    # the pools of all layers, one allocation each
    pools = {n: torch.stack([p[n] for p, _ in per_layer]) for n in per_layer[0][0]}
    # accepted: a prefix 0, 1, .. of the draft, then later tokens, behind all the kept rows'
    # places, so that moving them twice is moving them once
    rng = random.Random(seed)
    kept = torch.full((B, max(1, c["kept"])), -1, dtype=torch.int32)
    for b in range(B):
        m = c["kept"] if b % 2 == 0 else rng.randint(0, c["kept"])
        same = rng.randint(min(1, m), m)
        later = sorted(rng.sample(range(m, c["new"]), min(m - same, c["new"] - m)))
        path = list(range(same)) + later
        kept[b, :len(path)] = torch.tensor(path, dtype=torch.int32)
    return dict(kind="keep", bits=c["bits"], new=c["new"], page=c["page"], pools=pools,
                tables=torch.stack([t for _, t in per_layer]), kept=kept.to(DEV),
                lens=_i32([rows] * L), lens_out=torch.zeros((L, B), dtype=torch.int32, device=DEV))


_PREPARE = {"append8": _prepare_append8, "decode8": _prepare_decode8, "tree": _prepare_tree,
            "keep": _prepare_keep}


def prepare(case, seed):
    s = _PREPARE[case["kind"]](case, seed)
    s["held"] = _held(case.get("bits", 8), s["pools"])
    if own:
        # the handles that a serving program keeps for a layer's cache: pointers, strides, the
        # frequencies, scratch memory
        from paper_2608_08684_gb300 import ripple as R

        def cache(p, table):
            if case.get("bits", 8) != 8:
                return R.PagedCache(p["k"], p["v"], table)
            return R.PagedCache(p["k"], p["v"], table, k_scales=p["k_scales"],
                                v_scales=p["v_scales"], dtype=_DT[case["dtype"]])

        if s["kind"] == "keep":
            s["layers"] = R.KeepTables([cache({n: x[l] for n, x in s["held"].items()},
                                              s["tables"][l]) for l in range(case["layers"])])
            return s
        s["cache"] = cache(s["held"], s["table"])
        need = 0
        if s["kind"] == "append8":
            s["rope"] = R.Rope(s["inv_freq"], interleaved=s["inter"])
        elif s["kind"] == "decode8":
            need = R.ripple_paged_decode_workspace_bytes(s["cache"], case["q_heads"])
        else:
            need = R.ripple_paged_tree_workspace_bytes(s["cache"], case["q_heads"], s["most_new"])
        s["ws"] = torch.empty(need, dtype=torch.uint8, device=DEV)
    elif s["kind"] == "append8":
        s["inv_freq"] = torch.tensor(s["inv_freq"], dtype=torch.float64, device=DEV)
    return s


# ------------------------------------------------------------------ the plain forms


def _places(s):
    """(sequence, token of it, cache row, whether it has one) of every token."""
    t = torch.arange(s["n"], device=DEV)
    if s["starts"] is None:
        b = t // (s["n"] // s["B"])
        i, new = t - b * (s["n"] // s["B"]), s["n"] // s["B"]
        row = s["lens"][b] - new + i
    else:
        b = torch.searchsorted(s["starts"], t, right=True, out_int32=True) - 1
        i = t - s["starts"][b]
        row = s["lens"][b] - s["starts"][b + 1] + t
    return b.long(), i.long(), row.clamp(min=0).long(), row >= 0


def _rotate(x, cos, sin, rot, inter):
    x = x.float()
    if inter:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack((a, b), -1).flatten(-2) if inter else torch.cat((a, b), -1)
    return torch.cat((turned, x[..., rot:]), -1)


def _plain_append8(s):
    n, pools = s["n"], s["pools"]
    flat = lambda x: x.flatten(0, 1) if s["starts"] is None else x[:n]  # noqa: E731
    angle = flat(s["pos"][..., None])[:n].double() * s["inv_freq"]
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    b, _, row, valid = _places(s)
    page, slot = s["table"][b, row // s["page"]].long(), row % s["page"]
    keep = valid[:, None, None]
    k = _rotate(flat(s["k"]), cos, sin, s["rot"], s["inter"])
    for name, x in (("k", k), ("v", flat(s["v"]))):
        codes, scales = _quantise(x)
        to, to_scales = pools[name], pools[name + "_scales"]
        to[page, :, slot] = torch.where(keep, codes, to[page, :, slot])
        to_scales[page, :, slot] = torch.where(keep[..., 0], scales, to_scales[page, :, slot])
    q = _rotate(flat(s["q"]), cos, sin, s["rot"], s["inter"]).to(s["q_out"].dtype)
    if s["starts"] is None:
        s["q_out"].copy_(q.view(s["q_out"].shape))
    else:
        s["q_out"][:n] = q
    return {"q": s["q_out"], **s["held"]}


def _rows_of(s):
    """Every sequence's keys and values, [B][rows][heads][dims] in 32 bits."""
    r = torch.arange(max(1, s["most"]), device=DEV)
    page, slot = s["table"].clamp(min=0).long()[:, r // s["page"]], r % s["page"]
    p = s["pools"]
    if s["bits"] != 8:
        return [p[n][page, :, slot].float() for n in ("k", "v")]
    return [p[n][page, :, slot].view(torch.float8_e4m3fn).float()
            * _pow2(p[n + "_scales"][page, :, slot])[..., None] for n in ("k", "v")]


def _attend(q, k, v, there):
    """q [B][tokens][Hq][D], there [B][tokens][rows]: the outputs and the logs of the sums."""
    B, n, Hq, D = q.shape
    H = k.shape[2]
    q = q.float().view(B, n, H, -1, D)
    x = torch.einsum("bnhgd,brhd->bhgnr", q, k) / math.sqrt(D)
    x = torch.where(there[:, None, None], x, -math.inf)
    m = x.amax(4, keepdim=True)
    m = torch.where(torch.isinf(m), 0.0, m)
    p = torch.exp(x - m)
    total = p.sum(4, keepdim=True)
    lse = (m + torch.log(total))[..., 0].permute(0, 3, 1, 2).reshape(B, n, Hq)
    p = p / torch.where(total > 0, total, 1.0)
    return torch.einsum("bhgnr,brhd->bnhgd", p, v).reshape(B, n, Hq, D), lse


def _plain_decode8(s):
    k, v = _rows_of(s)
    there = torch.arange(k.shape[1], device=DEV)[None, None] < s["lens"][:, None, None]
    out, lse = _attend(s["q"][:, None], k, v, there)
    return {"out": out[:, 0], "lse": lse[:, 0]}


def _plain_tree(s):
    k, v = _rows_of(s)
    b, i, _, _ = _places(s)
    B, n, N = s["B"], s["n"], s["most_new"]
    lead = 2 if s["starts"] is None else 1
    q = torch.zeros((B, N) + s["q"].shape[lead:], dtype=s["q"].dtype, device=DEV)
    q[b, i] = s["q"].flatten(0, lead - 1)[:n]
    masks = torch.zeros((B, N), dtype=torch.int64, device=DEV)
    masks[b, i] = (torch.bitwise_left_shift(2, i) - 1 if s["masks"] is None
                   else s["masks"].flatten()[:n])
    new = n // B if s["starts"] is None else s["starts"].diff()
    j = torch.arange(k.shape[1], device=DEV)[None] - (s["lens"] - new)[:, None]
    seen = (masks[:, :, None] >> j.clamp(0, 63)[:, None] & 1) > 0
    in_cache = (j < (new if s["starts"] is None else new[:, None])) & (s["lens"] > 0)[:, None]
    out, lse = _attend(q, k, v, ((j < 0)[:, None] | seen) & in_cache[:, None])
    s["out"].view((-1,) + s["out"].shape[lead:])[:n] = out[b, i].to(s["out"].dtype)
    s["lse"].view(-1, s["lse"].shape[-1])[:n] = lse[b, i]
    return {"out": s["out"], "lse": s["lse"]}


def _plain_keep(s):
    kept = s["kept"].long()
    L, ps = s["lens"].shape[0], s["page"]
    first = (s["lens"] - s["new"]).long()[..., None]  # [L][B][1]
    j = torch.arange(kept.shape[1], device=DEV)
    src, dst = first + kept.clamp(min=0), first + j
    at = torch.arange(L, device=DEV)[:, None, None]
    b = torch.arange(kept.shape[0], device=DEV)[None, :, None]
    place = lambda row: (at, s["tables"][at, b, row // ps].long(), slice(None), row % ps)  # noqa: E731
    for x in s["pools"].values():
        row = x[place(src)]
        there = (kept >= 0)[None, :, :, None]
        x[place(dst)] = torch.where(there[..., None] if row.dim() == 5 else there, row, x[place(dst)])
    s["lens_out"].copy_(s["lens"] - s["new"] + (kept >= 0).sum(1))
    return {"lens": s["lens_out"], **s["held"]}


# ------------------------------------------------------------------ a pass


def run(s):
    if own:
        from paper_2608_08684_gb300 import ripple as R
        if s["kind"] == "append8":
            R.ripple_paged_append(s["cache"], s["lens"], s["k"], s["v"], rope=s["rope"],
                                  positions=s["pos"], seq_starts=s["starts"], q=s["q"],
                                  q_out=s["q_out"])
            return {"q": s["q_out"], **s["held"]}
        if s["kind"] == "decode8":
            R.ripple_paged_decode_attn(s["cache"], s["q"], s["lens"], s["out"], s["ws"],
                                       lse=s["lse"])
            return {"out": s["out"], "lse": s["lse"]}
        if s["kind"] == "tree":
            R.ripple_paged_tree_attn(s["cache"], s["q"], s["lens"], s["out"], s["ws"],
                                     masks=s["masks"], seq_starts=s["starts"],
                                     max_tokens=s["most_new"], lse=s["lse"])
            return {"out": s["out"], "lse": s["lse"]}
        R.ripple_paged_keep_rows(s["layers"], s["lens"], s["kept"], n_tokens=s["new"],
                                 lens_out=s["lens_out"])
        return {"lens": s["lens_out"], **s["held"]}
    return {"append8": _plain_append8, "decode8": _plain_decode8, "tree": _plain_tree,
            "keep": _plain_keep}[s["kind"]](s)


# ------------------------------------------------------------------ what a pass cannot do without


def work(case):
    c = case
    e = 4 if c["dtype"] == "f32" else 2
    new, rows = _lens(c)
    H, D, B = c["kv_heads"], c["dim"], c["batch"]
    bits = c.get("bits", 8)
    row = H * (D + 1) if bits == 8 else H * D * bits // 8  # bytes of a cache row's keys
    pages = sum(-(-r // c["page"]) for r in rows)
    if c["kind"] == "keep":
        # every second sequence keeps c["kept"] rows, the others half of it; about half move
        moved = c["layers"] * (B * c["kept"]) // 2
        return {"bytes": 2 * 2 * moved * row + 4 * B * (2 * c["layers"] + c["kept"]) + 8 * moved,
                "flops": 0}
    Hq = c["q_heads"]
    if c["kind"] == "append8":
        n = sum(new)
        return {"bytes": n * ((2 * Hq + 2 * H) * D * e + 2 * row + 8) + 4 * B,
                "flops": 3 * n * (Hq + H) * c["rot"] + 4 * n * H * D}
    if c["kind"] == "decode8":
        return {"bytes": 2 * sum(rows) * row + 4 * pages + B * (Hq * D * (e + 4) + 4 * Hq + 4),
                "flops": 4 * sum(rows) * Hq * D}
    n = sum(new)
    pairs = sum(m * (r - m) + m * (m + 1) // 2 for m, r in zip(new, rows) if r)
    return {"bytes": 2 * sum(rows) * row + 4 * pages + n * (2 * Hq * D * e + 4 * Hq + 8) + 8 * B,
            "flops": 4 * pairs * Hq * D}


# ------------------------------------------------------------------ the same in 64 bits


def _codes(x):
    """Rows in 64 bits as the values of their codes, and the values of their scales."""
    a = x.abs().amax(-1)
    e = torch.ceil(torch.log2(a / 448)).clamp(-120, 120)
    for _ in range(2):  # the logarithm's own rounding
        e = torch.where(a > 448 * torch.exp2(e), e + 1, torch.where(2 * a <= 448 * torch.exp2(e), e - 1, e))
    scale = torch.exp2(e.clamp(-120, 120))
    y = x / scale[..., None]
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step, scale


def _exact_append8(c, s):
    inv = torch.tensor(_inv_freq(c), dtype=torch.float64, device=DEV)
    half = c["rot"] // 2
    pairs = [(2 * j, 2 * j + 1) if c["inter"] else (j, j + half) for j in range(half)]
    first, second = (torch.tensor(p, device=DEV) for p in zip(*pairs))
    out = {"q": s["q_out"].double()}
    for n, x in s["pools"].items():
        out[n] = _pow2(x).double() if n.endswith("_scales") else x.view(torch.float8_e4m3fn).double()
    rows, ps = s["lens"].tolist(), c["page"]
    begin = s["starts"].tolist() if c["ragged"] else [b * c["new_lo"] for b in range(c["batch"] + 1)]
    tokens = {x: s[x] if c["ragged"] else s[x].flatten(0, 1) for x in ("q", "k", "v")}
    q_out, pos = out["q"].view(-1, c["q_heads"], c["dim"]), s["pos"].flatten()

    def turned(x, angle):
        y = x.double()
        a, b = y[..., first], y[..., second]
        y[..., first] = a * angle.cos() - b * angle.sin()
        y[..., second] = a * angle.sin() + b * angle.cos()
        return y

    for b in range(c["batch"]):
        t0, t1 = begin[b], begin[b + 1]
        angle = (pos[t0:t1, None].double() * inv)[:, None]
        q_out[t0:t1] = turned(tokens["q"][t0:t1], angle)
        if rows[b] == 0:
            continue
        at = torch.arange(rows[b] - (t1 - t0), rows[b], device=DEV)
        page = s["table"][b, at // ps].long()
        for n, x in (("k", turned(tokens["k"][t0:t1], angle)), ("v", tokens["v"][t0:t1].double())):
            out[n][page, :, at % ps], out[n + "_scales"][page, :, at % ps] = _codes(x)
    return out


def _cache64(c, s, b, n, h):
    """The first n keys and values of a sequence's head."""
    pages = s["table"][b, :-(-n // c["page"])].long()
    for name in ("k", "v"):
        x = s["pools"][name][pages, h]
        if s["bits"] == 8:
            x = x.view(torch.float8_e4m3fn).double()
            x = x * torch.exp2(s["pools"][name + "_scales"][pages, h].double() - 127)[..., None]
        yield x.reshape(-1, c["dim"])[:n].double()


def _exact_decode8(c, s):
    B, Hq, H, D = c["batch"], c["q_heads"], c["kv_heads"], c["dim"]
    out = torch.zeros((B, Hq, D), dtype=torch.float64, device=DEV)
    lse = torch.full((B, Hq), -math.inf, dtype=torch.float64, device=DEV)
    for b, n in enumerate(s["lens"].tolist()):
        for h in range(H if n else 0):
            k, v = _cache64(c, s, b, n, h)
            heads = slice(h * Hq // H, (h + 1) * Hq // H)
            x = s["q"][b, heads].double() @ k.T * D ** -0.5
            lse[b, heads] = torch.logsumexp(x, 1)
            out[b, heads] = torch.softmax(x, 1) @ v
    return {"out": out, "lse": lse}


def _exact_tree(c, s):
    Hq, H, D = c["q_heads"], c["kv_heads"], c["dim"]
    out, lse = s["out"].double(), s["lse"].double()
    flat_out, flat_lse = out.view(-1, Hq, D), lse.view(-1, Hq)
    q = s["q"].reshape(-1, Hq, D)
    new = s["n"] // s["B"] if s["starts"] is None else 0
    begin = [b * new for b in range(s["B"] + 1)] if s["starts"] is None else s["starts"].tolist()
    masks = None if s["masks"] is None else s["masks"].flatten().tolist()
    for b, n in enumerate(s["lens"].tolist()):
        t0, t1 = begin[b], begin[b + 1]
        m = t1 - t0
        if n == 0:
            flat_out[t0:t1], flat_lse[t0:t1] = 0.0, -math.inf
            continue
        hidden = torch.tensor([[j > i if masks is None else not masks[t0 + i] >> j & 1
                                for j in range(m)] for i in range(m)], device=DEV)
        for h in range(H):
            k, v = _cache64(c, s, b, n, h)
            heads = slice(h * Hq // H, (h + 1) * Hq // H)
            x = q[t0:t1, heads].double() @ k.T * D ** -0.5
            x[:, :, n - m:].masked_fill_(hidden[:, None], -math.inf)
            flat_lse[t0:t1, heads] = torch.logsumexp(x, 2)
            flat_out[t0:t1, heads] = torch.softmax(x, 2) @ v
    return {"out": out, "lse": lse}


def _exact_keep(c, s):
    out = {n: x.clone() for n, x in s["held"].items()}
    lens_out, kept, ps = s["lens_out"].clone(), s["kept"].tolist(), c["page"]
    tables = s["tables"].tolist()
    for l, lens in enumerate(s["lens"].tolist()):
        src, dst = [], []
        for b, n in enumerate(lens):
            path = [x for x in kept[b] if x >= 0]
            lens_out[l, b] = n - c["new"] + len(path)
            for j, x in enumerate(path):
                for rows, r in ((src, n - c["new"] + x), (dst, n - c["new"] + j)):
                    rows.append((tables[l][b][r // ps], r % ps))
        if src:
            (sp, ss), (dp, ds) = (torch.tensor(x, device=DEV).T for x in (src, dst))
            for n, x in s["pools"].items():
                out[n].view(x.dtype)[l, dp, :, ds] = x[l, sp, :, ss]
    return {"lens": lens_out, **out}


def exact(case, seed):
    s = _PREPARE[case["kind"]](case, seed)
    s["held"] = _held(case.get("bits", 8), s["pools"])
    return {"append8": _exact_append8, "decode8": _exact_decode8, "tree": _exact_tree,
            "keep": _exact_keep}[case["kind"]](case, s)

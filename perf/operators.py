"""The operators of a decode step over a paged KV cache, as a serving program calls them.

  append    new tokens' keys and values into a paged cache, rotated on the way, with
            the queries rotated in the same pass (a decode step's tokens, the ragged
            chunks of a prefill, whole prompts)
  decode    attention of one new token per sequence over the paged cache
  logprobs  log probabilities of given tokens, the entropy of each position and the
            top alternatives, from logits over the vocabulary

With `own` false the operators are computed in their plain form: elementary torch
operations in 32 bits (angles in 64), rounded once at the end. `exact` computes the
same from the definitions in 64 bits, one sequence or a few rows at a time.

Shapes are those of the repository's synthetic workloads (8B: 32 query and 8 KV heads
of 128 dims; 70B: 64 and 8; a 128256-token vocabulary; caches of a few hundred rows
after compression up to 128k uncompressed ones) and of odd sizes between them. Keys
are N(0, 1) with a per-channel lognormal(0, 0.5) scale, values N(0, 1), queries
N(0, 1) with a gain of 2 (attention as peaked as a trained model's), logits
2.5 N(0, 1) with four likely tokens a position.
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
        # one token of one sequence, after the fused projection of its q, k and v
        dict(name="append_token", kind="append", dtype="bf16", q_heads=32, kv_heads=8, dim=128,
             page=16, rot=128, inter=False, batch=1, new_lo=1, new_hi=1, old_lo=900, old_hi=900,
             idle=0, ragged=False, layout="heads", mix=1),
        # a decode step of a batch padded for a captured graph (12 sequences idle)
        dict(name="append_batch", kind="append", dtype="bf16", q_heads=64, kv_heads=8, dim=128,
             page=32, rot=128, inter=False, batch=108, new_lo=1, new_hi=1, old_lo=1,
             old_hi=131071, idle=12, ragged=False, layout="heads", mix=2),
        # prefill chunks of a few sequences, fp32, half of the dims rotated in adjacent pairs
        dict(name="append_chunk_f32", kind="append", dtype="f32", q_heads=14, kv_heads=2, dim=64,
             page=8, rot=32, inter=True, batch=5, new_lo=1, new_hi=1500, old_lo=1, old_hi=5000,
             idle=0, ragged=True, layout="rows", mix=3),
        # whole prompts
        dict(name="append_prompts", kind="append", dtype="bf16", q_heads=32, kv_heads=8, dim=128,
             page=64, rot=128, inter=False, batch=6, new_lo=4000, new_hi=16384, old_lo=1,
             old_hi=300, idle=0, ragged=True, layout="heads", mix=4),
        # one sequence over a compressed cache
        dict(name="decode_short", kind="decode", dtype="bf16", q_heads=32, kv_heads=8, dim=128,
             page=16, batch=1, lo=470, hi=470, layout="heads", mix=5),
        # one sequence at 128k tokens, eight query heads a KV head
        dict(name="decode_128k_g8", kind="decode", dtype="bf16", q_heads=64, kv_heads=8, dim=128,
             page=64, batch=1, lo=131055, hi=131055, layout="heads", mix=6),
        # continuous batching: 64 sequences, from an idle one to 32k tokens
        dict(name="decode_ragged", kind="decode", dtype="bf16", q_heads=32, kv_heads=8, dim=128,
             page=16, batch=64, lo=64, hi=32768, layout="heads", mix=7),
        # fp32, seven query heads a KV head, the heads of a row side by side
        dict(name="decode_f32_g7", kind="decode", dtype="f32", q_heads=28, kv_heads=4, dim=64,
             page=32, batch=9, lo=100, hi=6000, layout="rows", mix=8),
        # the token just sampled, with its alternatives
        dict(name="logprobs_token", kind="logprobs", dtype="bf16", rows=1, vocab=128256, top=5,
             masked=0.0, scale=1.0, mix=9),
        # a batch's sampled tokens, at a temperature
        dict(name="logprobs_batch", kind="logprobs", dtype="f32", rows=64, vocab=128256, top=20,
             masked=0.0, scale=1.25, mix=10),
        # scoring given texts
        dict(name="logprobs_texts", kind="logprobs", dtype="bf16", rows=2048, vocab=128256, top=1,
             masked=0.0, scale=1.0, mix=11),
        # a grammar's mask (most tokens at -infinity), an odd vocabulary, no alternatives
        dict(name="logprobs_masked", kind="logprobs", dtype="f32", rows=333, vocab=32003, top=0,
             masked=0.9, scale=1.0, mix=12),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


# (query heads, KV heads, head dim)
_HEADS = [(32, 8, 128), (32, 8, 128), (64, 8, 128), (28, 4, 128), (8, 8, 64), (40, 4, 64),
          (5, 1, 128), (16, 1, 64)]


def draw(rng):
    kind = rng.choice(["append", "append", "decode", "decode", "logprobs"])
    mix = rng.randrange(1, 1 << 30)
    if kind == "logprobs":
        vocab = _log(rng, 1000, 262144)
        return dict(kind=kind, dtype=rng.choice(["bf16", "f32"]), vocab=vocab,
                    rows=_log(rng, 1, min(4096, 131_000_000 // vocab)),
                    top=rng.choice([0, 1, 5, 20, 32]), masked=rng.choice([0.0, 0.0, 0.9]),
                    scale=rng.choice([1.0, 1.0, 0.7, 1.25]), mix=mix)
    hq, hkv, dim = rng.choice(_HEADS)
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    c = dict(kind=kind, dtype=dtype, q_heads=hq, kv_heads=hkv, dim=dim,
             page=rng.choice([1, 8, 16, 16, 32, 64, 128, 256]),
             layout=rng.choice(["heads", "heads", "rows"]), mix=mix)
    if kind == "append":
        c["rot"] = rng.choice([dim, dim, dim, dim // 2])
        c["inter"] = rng.choice([False, False, True])
        c["ragged"] = rng.choice([False, True])
        if c["ragged"]:
            c["batch"] = _log(rng, 1, 16)
            most = 44_000 * 6144 // ((hq + 2 * hkv) * dim * (2 if dtype == "f32" else 1))
            c["new_hi"] = _log(rng, 16, min(16384, most // c["batch"]))
            c["new_lo"] = _log(rng, 1, c["new_hi"])
        else:
            c["batch"] = _log(rng, 1, 256)
            c["new_lo"] = c["new_hi"] = rng.choice([1, 1, 1, 4])
        c["old_lo"], c["old_hi"] = 1, _log(rng, 16, 131072 // max(1, c["batch"] // 16))
        c["idle"] = 0 if c["ragged"] or c["batch"] < 4 else rng.choice([0, c["batch"] // 8])
        return c
    c["batch"] = _log(rng, 1, 256)
    # at most about the bytes of the largest listed steps, also if every sequence were the longest
    e = 4 if dtype == "f32" else 2
    most = min(131072, 1_250_000_000 // (2 * e * hkv * dim * c["batch"]))
    c["hi"] = _log(rng, 16, most)
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
    their order. A decode batch of eight or more has an empty sequence and one of one row."""
    c, rng = case, random.Random(case["mix"])
    if c["kind"] == "decode":
        rows = [_log(rng, c["lo"], c["hi"]) for _ in range(c["batch"])]
        if c["batch"] >= 8:
            rows[:2] = [0, 1]
        return [1] * c["batch"], rows
    new = [_log(rng, c["new_lo"], c["new_hi"]) for _ in range(c["batch"])]
    rows = [n + _log(rng, c["old_lo"], c["old_hi"]) for n in new]
    for b in range(c["idle"]):
        rows[c["batch"] - 1 - b] = 0
    return new, rows


def _pools(c, seed, rows, fill):
    """Pages for `rows` rows of every sequence, handed out in random order, and the table.
    Entries behind a sequence's last page are no pages."""
    ps, H, D, dt = c["page"], c["kv_heads"], c["dim"], _DT[c["dtype"]]
    need = [max(1, -(-n // ps)) for n in rows]
    n_pages, width = sum(need), max(need)
    perm = torch.randperm(n_pages, device=DEV, generator=_gen(seed, 20)).to(torch.int32)
    starts = [0]
    for n in need:
        starts.append(starts[-1] + n)
    at = _i32(starts[:-1])[:, None] + torch.arange(width, device=DEV)[None]
    table = perm[at.clamp(max=n_pages - 1)]
    table = torch.where(torch.arange(width, device=DEV)[None] < _i32(need)[:, None], table, -1)
    # heads: [page][head][row][dim]; rows: [page][row][head][dim]
    shape = (n_pages, H, ps, D) if c["layout"] == "heads" else (n_pages, ps, H, D)
    if fill:
        scale = torch.exp(0.5 * _randn((H, D), torch.float32, seed, 21)).to(dt)
        k, v = _randn(shape, dt, seed, 22), _randn(shape, dt, seed, 23)
        k.mul_(scale[:, None] if c["layout"] == "heads" else scale)
    else:
        k, v = (torch.zeros(shape, dtype=dt, device=DEV) for _ in range(2))
    if c["layout"] == "rows":
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    return k, v, table.contiguous()


def _inv_freq(c):
    """Base 500000, the usual spacing."""
    return [500000.0 ** (-2.0 * j / c["rot"]) for j in range(c["rot"] // 2)]


def _prepare_append(c, seed):
    new, rows = _lens(c)
    order = list(range(c["batch"]))
    random.Random(seed).shuffle(order)
    new, rows = [new[i] for i in order], [rows[i] for i in order]
    B, Hq, H, D, dt = c["batch"], c["q_heads"], c["kv_heads"], c["dim"], _DT[c["dtype"]]
    k_pages, v_pages, table = _pools(c, seed, rows, False)
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
    starts = [0]
    for m in new:
        starts.append(starts[-1] + m)
    return dict(kind="append", n=n, B=B, page=c["page"], rot=c["rot"], inter=c["inter"],
                inv_freq=_inv_freq(c), q=q, k=k, v=v, q_out=q_out, pos=pos.view(q.shape[:-2]),
                starts=_i32(starts) if c["ragged"] else None, lens=_i32(rows), k_pages=k_pages,
                v_pages=v_pages, table=table)


def _prepare_decode(c, seed):
    _, rows = _lens(c)
    random.Random(seed).shuffle(rows)
    B, Hq, D, dt = c["batch"], c["q_heads"], c["dim"], _DT[c["dtype"]]
    k_pages, v_pages, table = _pools(c, seed, rows, True)
    return dict(kind="decode", most=max(rows), page=c["page"], lens=_i32(rows), k_pages=k_pages,
                v_pages=v_pages, table=table, q=_randn((B, Hq, D), dt, seed, 3).mul_(2),
                out=torch.zeros((B, Hq, D), device=DEV), lse=torch.zeros((B, Hq), device=DEV))


def _prepare_logprobs(c, seed):
    n, V = c["rows"], c["vocab"]
    x = _randn((n, V), torch.float32, seed, 2).mul_(2.5)
    likely = torch.randint(0, V, (n, 4), device=DEV, generator=_gen(seed, 3))
    x.scatter_add_(1, likely, torch.full(likely.shape, 12.0, device=DEV))
    if c["masked"]:
        hide = torch.rand((n, V), device=DEV, generator=_gen(seed, 4)) < c["masked"]
        hide.scatter_(1, likely, False)
        x.masked_fill_(hide, -math.inf)
    # mostly a likely token, some from anywhere the mask allows
    other = torch.randint(0, V, (n,), device=DEV, generator=_gen(seed, 5))
    rows = torch.arange(n, device=DEV)
    pick = (rows % 4 == 3) & torch.isfinite(x[rows, other])
    tokens = torch.where(pick, other, likely[:, 0]).to(torch.int32)
    s = dict(kind="logprobs", logits=x.to(_DT[c["dtype"]]), tokens=tokens, top=c["top"],
             scale=c["scale"], logprob=torch.zeros(n, device=DEV), entropy=torch.zeros(n, device=DEV))
    if c["top"]:
        s["top_idx"] = torch.zeros((n, c["top"]), dtype=torch.int32, device=DEV)
        s["top_logprob"] = torch.zeros((n, c["top"]), device=DEV)
    return s


def prepare(case, seed):
    s = {"append": _prepare_append, "decode": _prepare_decode,
         "logprobs": _prepare_logprobs}[case["kind"]](case, seed)
    if own and s["kind"] != "logprobs":
        # the handles that a serving program keeps for a layer's cache: pointers, strides, the
        # frequencies, scratch memory
        from paper_2608_08684_gb300 import ripple as R
        s["cache"] = R.PagedCache(s["k_pages"], s["v_pages"], s["table"])
        if s["kind"] == "append":
            s["rope"] = R.Rope(s["inv_freq"], interleaved=s["inter"])
        else:
            s["ws"] = torch.empty(R.ripple_paged_decode_workspace_bytes(s["cache"], case["q_heads"]),
                                  dtype=torch.uint8, device=DEV)
    elif s["kind"] == "append":
        s["inv_freq"] = torch.tensor(s["inv_freq"], dtype=torch.float64, device=DEV)
    return s


# ------------------------------------------------------------------ the plain forms


def _places(s):
    """(sequence, cache row, whether it has one) of every token."""
    t = torch.arange(s["n"], device=DEV)
    if s["starts"] is None:
        b = t // (s["n"] // s["B"])
        i, new = t - b * (s["n"] // s["B"]), s["n"] // s["B"]
        row = s["lens"][b] - new + i
    else:
        b = torch.searchsorted(s["starts"], t, right=True, out_int32=True) - 1
        row = s["lens"][b] - s["starts"][b + 1] + t
    return b.long(), row.clamp(min=0).long(), row >= 0


def _rotate(x, cos, sin, rot, inter):
    x = x.float()
    if inter:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack((a, b), -1).flatten(-2) if inter else torch.cat((a, b), -1)
    return torch.cat((turned, x[..., rot:]), -1)


def _plain_append(s):
    n = s["n"]
    flat = lambda x: x.flatten(0, 1) if s["starts"] is None else x[:n]  # noqa: E731
    angle = flat(s["pos"][..., None])[:n].double() * s["inv_freq"]
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    b, row, valid = _places(s)
    page, slot = s["table"][b, row // s["page"]].long(), row % s["page"]
    dt = s["k_pages"].dtype
    k = _rotate(flat(s["k"]), cos, sin, s["rot"], s["inter"]).to(dt)
    keep = valid[:, None, None]
    s["k_pages"][page, :, slot] = torch.where(keep, k, s["k_pages"][page, :, slot])
    s["v_pages"][page, :, slot] = torch.where(keep, flat(s["v"]), s["v_pages"][page, :, slot])
    q = _rotate(flat(s["q"]), cos, sin, s["rot"], s["inter"]).to(dt)
    if s["starts"] is None:
        s["q_out"].copy_(q.view(s["q_out"].shape))
    else:
        s["q_out"][:n] = q
    return {"q": s["q_out"], "k": s["k_pages"], "v": s["v_pages"]}


def _plain_decode(s):
    most = max(1, s["most"])
    r = torch.arange(most, device=DEV)
    page, slot = s["table"].clamp(min=0).long()[:, r // s["page"]], r % s["page"]
    k, v = s["k_pages"][page, :, slot], s["v_pages"][page, :, slot]  # [B][rows][heads][dims]
    B, _, H, D = k.shape
    q = s["q"].float().view(B, H, -1, D)
    x = torch.einsum("bhgd,brhd->bhgr", q, k.float()) / math.sqrt(D)
    there = (r[None] < s["lens"][:, None])[:, None, None]
    x = torch.where(there, x, -math.inf)
    m = x.amax(3, keepdim=True)
    m = torch.where(torch.isinf(m), 0.0, m)
    p = torch.exp(x - m)
    total = p.sum(3, keepdim=True)
    lse = (m + torch.log(total)).reshape(B, -1)
    p = p / torch.where(total > 0, total, 1.0)
    return {"out": torch.einsum("bhgr,brhd->bhgd", p, v.float()).reshape(B, -1, D), "lse": lse}


def _plain_logprobs(s):
    raw = s["logits"].float()
    x = raw * s["scale"]
    d = x - x.amax(1, keepdim=True)
    w = torch.exp(d)
    total = w.sum(1)
    log_total = torch.log(total)
    out = {"logprob": d.gather(1, s["tokens"].long()[:, None])[:, 0] - log_total,
           "entropy": log_total - torch.where(w > 0, w * d, 0.0).sum(1) / total}
    if s["top"]:
        at = torch.sort(raw, dim=1, descending=True, stable=True).indices[:, :s["top"]]
        out["top_idx"] = at.to(torch.int32)
        out["top_logprob"] = d.gather(1, at) - log_total[:, None]
    return out


# ------------------------------------------------------------------ a pass


def run(s):
    if own:
        from paper_2608_08684_gb300 import ripple as R
        if s["kind"] == "append":
            R.ripple_paged_append(s["cache"], s["lens"], s["k"], s["v"], rope=s["rope"],
                                  positions=s["pos"], seq_starts=s["starts"], q=s["q"],
                                  q_out=s["q_out"])
            return {"q": s["q_out"], "k": s["k_pages"], "v": s["v_pages"]}
        if s["kind"] == "decode":
            R.ripple_paged_decode_attn(s["cache"], s["q"], s["lens"], s["out"], s["ws"],
                                       lse=s["lse"])
            return {"out": s["out"], "lse": s["lse"]}
        R.ripple_token_logprobs(s["logits"], s["tokens"], s["logprob"], entropy_out=s["entropy"],
                                top_idx=s.get("top_idx"), top_logprob=s.get("top_logprob"),
                                scale=s["scale"])
        return {k: s[k] for k in ("logprob", "entropy", "top_idx", "top_logprob") if k in s}
    return {"append": _plain_append, "decode": _plain_decode,
            "logprobs": _plain_logprobs}[s["kind"]](s)


# ------------------------------------------------------------------ what a pass cannot do without


def work(case):
    c = case
    e = 4 if c["dtype"] == "f32" else 2
    if c["kind"] == "logprobs":
        n, V = c["rows"], c["vocab"]
        return {"bytes": n * (V * e + 12 + 8 * c["top"]), "flops": 4 * n * V}
    new, rows = _lens(c)
    Hq, H, D = c["q_heads"], c["kv_heads"], c["dim"]
    pages = sum(-(-r // c["page"]) for r in rows)
    if c["kind"] == "append":
        n = sum(new)
        return {"bytes": n * (2 * (Hq + 2 * H) * D * e + 8) + 4 * c["batch"],
                "flops": 3 * n * (Hq + H) * c["rot"]}
    return {"bytes": 2 * sum(rows) * H * D * e + 4 * pages
            + c["batch"] * (Hq * D * (e + 4) + 4 * Hq + 4),
            "flops": 4 * sum(rows) * Hq * D}


# ------------------------------------------------------------------ the same in 64 bits


def _exact_append(c, s):
    inv = torch.tensor(_inv_freq(c), dtype=torch.float64, device=DEV)
    half = c["rot"] // 2
    pairs = [(2 * j, 2 * j + 1) if c["inter"] else (j, j + half) for j in range(half)]
    first, second = (torch.tensor(p, device=DEV) for p in zip(*pairs))
    out = {"q": s["q_out"].double(), "k": s["k_pages"].double(), "v": s["v_pages"].double()}
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
        out["k"][page, :, at % ps] = turned(tokens["k"][t0:t1], angle)
        out["v"][page, :, at % ps] = tokens["v"][t0:t1].double()
    return out


def _exact_decode(c, s):
    B, Hq, H, D = c["batch"], c["q_heads"], c["kv_heads"], c["dim"]
    out = torch.zeros((B, Hq, D), dtype=torch.float64, device=DEV)
    lse = torch.full((B, Hq), -math.inf, dtype=torch.float64, device=DEV)
    for b, n in enumerate(s["lens"].tolist()):
        if n == 0:
            continue
        pages = s["table"][b, :-(-n // c["page"])].long()
        for h in range(H):
            k, v = (x[pages, h].reshape(-1, D)[:n].double() for x in (s["k_pages"], s["v_pages"]))
            heads = slice(h * Hq // H, (h + 1) * Hq // H)
            x = s["q"][b, heads].double() @ k.T * D ** -0.5
            lse[b, heads] = torch.logsumexp(x, 1)
            out[b, heads] = torch.softmax(x, 1) @ v
    return {"out": out, "lse": lse}


def _exact_logprobs(c, s):
    logprob, entropy, top = [], [], []
    for i in range(0, c["rows"], 256):
        lp = torch.log_softmax(s["logits"][i:i + 256].double() * c["scale"], 1)
        logprob.append(lp.gather(1, s["tokens"][i:i + 256].long()[:, None])[:, 0])
        entropy.append(torch.special.entr(lp.exp()).sum(1))
        if c["top"]:
            top.append(lp.topk(c["top"], 1).values)
    out = {"logprob": torch.cat(logprob), "entropy": torch.cat(entropy)}
    if c["top"]:
        out |= {"top_idx": None, "top_logprob": torch.cat(top)}
    return out


def exact(case, seed):
    s = {"append": _prepare_append, "decode": _prepare_decode,
         "logprobs": _prepare_logprobs}[case["kind"]](case, seed)
    return {"append": _exact_append, "decode": _exact_decode,
            "logprobs": _exact_logprobs}[case["kind"]](case, s)

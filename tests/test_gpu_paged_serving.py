"""The paged operators together, as a serving program uses them: a prompt's layers compressed
to their budgets, the kept rows put into pages, decode steps of PagedDecodeLoop replayed from
a graph (an idle place in the batch), and the log probabilities of the tokens at its end.
Every step's attention against the oracle over the rows as they are stored, the stored rows
against the rotation in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import ripple_oracle as O
from paper_2608_08684_gb300 import synth
from paper_2608_08684_gb300.serving import PagedDecodeLoop
from tests import gpu_common as C
from tests import paged_common as P
from tests.test_gpu_logprobs import _check as check_logprobs

pytestmark = pytest.mark.gpu
DEV = "cuda"
STEPS, VOCAB = 5, 5003


def test_compress_to_pages_and_decode(lib):
    wl = synth.WORKLOADS["tiny"].replace(n_layers=3, batch=2, n_q_heads=8, n_kv_heads=2,
                                         head_dim=128, seq_len=700, dtype="bf16",
                                         kv_dist="scaled_sinks", seed=91)
    L, B, Hq, H, d, dt, page = 3, 3, 8, 2, 128, torch.bfloat16, 16  # a third, idle sequence
    G = Hq // H
    rng = np.random.default_rng(4)
    budgets = [60, 333, 150]
    inv = [10000.0 ** (-2.0 * j / d) for j in range(d // 2)]
    rope = lib.Rope(inv)
    caches, kept = [], []
    for l in range(L):
        q_win, k, v = (t.to(DEV) for t in C.layer_inputs(wl, l, "cpu"))
        out = C.run_compress(lib, wl, budgets[l], q_win, k, v, cap_extra=3)
        n = out["n"]
        kept.append(n)
        pages = -(-(n + STEPS + 1) // page)
        kp = P.randn((2 * pages + 3, H, page, d), "bf16", 900 + l)
        vp = P.randn((2 * pages + 3, H, page, d), "bf16", 950 + l)
        table = np.full((B, pages), -1, np.int32)
        table[:2] = rng.permutation(2 * pages + 3)[:2 * pages].reshape(2, pages)
        cache = lib.PagedCache(kp, vp, torch.from_numpy(table).to(DEV))
        # the kept rows, rotated already, into the pages of the two sequences
        two = lib.PagedCache(kp, vp, torch.from_numpy(table[:2].copy()).to(DEV))
        lib.ripple_paged_append(two, P.i32([n, n]), out["k_out"][:, :, :n].transpose(1, 2),
                                out["v_out"][:, :, :n].transpose(1, 2))
        caches.append((cache, kp, vp, table))
        for b in range(2):
            for which, pool in (("k_out", kp), ("v_out", vp)):
                rows = pool[torch.from_numpy(table[b].astype(np.int64)).to(DEV)]
                rows = rows.transpose(0, 1).reshape(H, -1, d)[:, :n]
                assert torch.equal(rows, out[which][b, :, :n])

    g = P.gen(5)
    wqkv = [(torch.randn(Hq * d, (Hq + 2 * H) * d, generator=g, device=DEV) / 32).to(dt) for _ in range(L)]
    wo = [(torch.randn(Hq * d, Hq * d, generator=g, device=DEV) / 32).to(dt) for _ in range(L)]
    wv = (torch.randn(Hq * d, VOCAB, generator=g, device=DEV) / 8).to(dt)
    hidden = torch.randn(B, Hq * d, generator=g, device=DEV).to(dt)
    qkv = [torch.zeros(B, Hq + 2 * H, d, dtype=dt, device=DEV) for _ in range(L)]
    rotated = [torch.zeros(B, Hq, d, dtype=dt, device=DEV) for _ in range(L)]
    logits = torch.zeros(B, VOCAB, dtype=dt, device=DEV)
    tokens = P.i32([0, 0, 0])
    answers = dict(logprob=torch.zeros(B, device=DEV), entropy=torch.zeros(B, device=DEV), lse=None,
                   idx=torch.zeros(B, 4, dtype=torch.int32, device=DEV),
                   top=torch.zeros(B, 4, device=DEV))

    def before(l):
        h = hidden.float()
        h = (h * torch.rsqrt(h.square().mean(-1, keepdim=True) + 1e-6)).to(dt)
        torch.mm(h, wqkv[l], out=qkv[l].view(B, -1))
        return qkv[l][:, :Hq], qkv[l][:, Hq:Hq + H], qkv[l][:, Hq + H:]  # views, strided

    def after(l, out):
        rotated[l].copy_(loop.q)
        hidden.add_(out.reshape(B, -1).to(dt) @ wo[l])
        if l == L - 1:  # the token taken, its log probability and the alternatives
            torch.mm(hidden, wv, out=logits)
            tokens.copy_(logits.argmax(1))
            lib.ripple_token_logprobs(logits, tokens, answers["logprob"],
                                      entropy_out=answers["entropy"], top_idx=answers["idx"],
                                      top_logprob=answers["top"], dev_status=loop.status)

    lens = P.i32([[n, n, 0] for n in kept])
    positions = P.i32([wl.seq_len, wl.seq_len, 0])
    loop = PagedDecodeLoop([c[0] for c in caches], lens, positions, P.i32([1, 1, 0]), Hq, rope,
                           before, after)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for step in range(STEPS):
            if step == 0:
                loop.issue_step()
            elif step == 1:
                loop.capture()
            if step > 0:
                loop.replay()
            s.synchronize()
            assert int(loop.status.item()) == 0
            assert lens.tolist() == [[n + step + 1] * 2 + [0] for n in kept]
            assert positions.tolist() == [wl.seq_len + step + 1] * 2 + [0]
            for l, (cache, kp, vp, table) in enumerate(caches):
                assert (loop.out[l][2] == 0).all()
                pos = [wl.seq_len + step] * 2
                for b in range(2):
                    n = kept[l] + step + 1
                    rows = [torch.stack([pool[table[b, r // page], :, r % page] for r in range(n)], 1)
                            for pool in (kp, vp)]
                    # the new row: rotated within the rounding to bf16 (2^-8), the values as given
                    x = synth.to_f64(qkv[l][b, Hq:Hq + H])
                    turned = O.rotate(x[None], pos[:1], inv)[0]
                    # within half a step of bf16 of the rotated value, and of |a| + |b| in fp32
                    bound = 2.0 ** -8 * np.abs(turned) + 2.0 ** -21 * np.abs(x).max()
                    assert (np.abs(synth.to_f64(rows[0][:, -1]) - turned) <= bound).all()
                    assert torch.equal(rows[1][:, -1], qkv[l][b, Hq + H:])
                    q = synth.to_f64(rotated[l][b])
                    for h in range(H):
                        ref = O.decode_attention(q[h * G:(h + 1) * G], synth.to_f64(rows[0][h]),
                                                 synth.to_f64(rows[1][h]), d ** -0.5)
                        C.assert_decode_close(loop.out[l][b, h * G:(h + 1) * G].cpu().numpy(), ref)
            check_logprobs(answers, logits, tokens, 4)
            assert torch.equal(answers["idx"][:, 0].long(), tokens.long()) or \
                (logits.gather(1, tokens.long()[:, None])[:, 0] == logits.amax(1)).all()

"""Drafted tokens as a serving program uses them: PagedDraftLoop's step (append, attention of
the tree) and keep, issued and replayed from graphs, over bf16, fp32 and 8-bit caches with an
idle place in the batch, then a decode step over what was kept. Every output against attention
in 64 bits over the rows as they are stored; kept rows byte for byte."""
import numpy as np
import pytest
import torch

from paper_2608_08684_gb300.serving import PagedDecodeLoop, PagedDraftLoop
from tests import gpu_common as C
from tests import paged8_common as P8
from tests import paged_common as P

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _rows(pool, b, n):
    """The first n rows as they are stored: [tensor][n][heads][..]."""
    at = [pool.place(b, r) for r in range(n)]
    p, s = (torch.tensor(x, device=DEV) for x in zip(*at))
    return [getattr(pool, x)[p, :, s].clone() for x in ("k", "v", "ks", "vs") if hasattr(pool, x)]


@pytest.mark.parametrize("kind", ["bf16", "q8-bf16", "f32"])
@pytest.mark.parametrize("tree", [True, False])
def test_drafts_kept_and_decoded_on(lib, kind, tree):
    L, B, n, Hq, H, d, page, room = 2, 3, 7, 8, 2, 128, 16, 200
    dt = P.DT[P8.type_of(kind)]
    pools = [P8.any_pool(lib, kind, [room, room, room], H, d, page, 30 + l) for l in range(L)]
    base = [[100, 0, 41], [64, 0, 3]]  # the second place of the batch is idle
    lens = P.i32(base)
    active = P.i32([1, 0, 1])
    positions = torch.zeros(B, n, dtype=torch.int32, device=DEV)
    masks = torch.zeros(B, n, dtype=torch.int64, device=DEV) if tree else None
    kept = torch.full((B, 4), -1, dtype=torch.int32, device=DEV)
    qkv = [torch.zeros(B, n, Hq + 2 * H, d, dtype=dt, device=DEV) for _ in range(L)]
    turned = [torch.zeros(B, n, Hq, d, dtype=dt, device=DEV) for _ in range(L)]
    rope = lib.Rope([10000.0 ** (-2.0 * j / d) for j in range(d // 2)])

    def before(l):
        return qkv[l][:, :, :Hq], qkv[l][:, :, Hq:Hq + H], qkv[l][:, :, Hq + H:]

    def after(l, out):
        turned[l].copy_(loop.q)

    loop = PagedDraftLoop([p.cache for p in pools], lens, positions, active, Hq, rope, before, after,
                          kept, masks)
    have = [list(x) for x in base]  # rows before the draft
    paths = [[[0, 2, 5], [], [1, 3, 4, 6]], [[], [], [0]], [[0, 1, 2, 3], [], [6]], [[3], [], [0, 6]]]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for step, path in enumerate(paths):
            for l in range(L):
                qkv[l].copy_(P.randn(qkv[l].shape, P8.type_of(kind), 100 + 10 * step + l))
            positions.copy_(torch.randint(0, 5000, (B, n), generator=P.gen(step), device=DEV).int())
            bits = P8.random_masks([n] * B, step) if tree else None
            if tree:
                masks.copy_(P8.to_i64(bits).view(B, n))
            kept.copy_(P.i32([p + [-1] * (4 - len(p)) for p in path]))
            if step == 0:
                loop.issue_step()
            elif step == 1:
                loop.capture()
            if step > 0:
                loop.replay()
            s.synchronize()
            assert int(loop.status.item()) == 0
            assert lens.tolist() == [[x + n if b != 1 else 0 for b, x in enumerate(row)] for row in have]
            for l in range(L):
                now = lens[l].tolist()
                out = loop.out[l]
                assert (out[1] == 0).all()
                want, _, size = P8.tree_ref(pools[l], turned[l].reshape(B * n, Hq, d), now, [n] * B, bits)
                got = out.double().cpu().numpy().reshape(want.shape)
                bound = C.DECODE_PREC_ATOL * max(1.0, np.abs(want).max())
                if dt is torch.bfloat16:
                    bound = bound + 2.0 ** -8 * (size + np.abs(want))
                assert (np.abs(got - want) <= bound).all()
            stored = [[_rows(pools[l], b, have[l][b] + n) if b != 1 else None for b in range(B)]
                      for l in range(L)]
            loop.issue_keep() if step == 0 else loop.replay_keep()
            s.synchronize()
            assert int(loop.status.item()) == 0
            for l in range(L):
                for b in (0, 2):
                    pre, m = have[l][b], len(path[b])
                    rows = list(range(pre)) + [pre + x for x in path[b]]
                    now = _rows(pools[l], b, pre + m)
                    for x, was in zip(now, stored[l][b]):
                        assert torch.equal(x, was[rows])
                    have[l][b] = pre + m
            assert lens.tolist() == have
        # an ordinary decode step over what is there
        one = [torch.zeros(B, Hq + 2 * H, d, dtype=dt, device=DEV).copy_(q[:, 0]) for q in qkv]
        dec_turned = [torch.zeros(B, Hq, d, dtype=dt, device=DEV) for _ in range(L)]
        dec = PagedDecodeLoop([p.cache for p in pools], lens, P.i32([300, 0, 300]), active, Hq, rope,
                              lambda l: (one[l][:, :Hq], one[l][:, Hq:Hq + H], one[l][:, Hq + H:]),
                              lambda l, out: dec_turned[l].copy_(dec.q))
        dec.issue_step()
        s.synchronize()
        assert int(dec.status.item()) == 0
        for l in range(L):
            now = [x + (b != 1) for b, x in enumerate(have[l])]
            assert lens[l].tolist() == now
            want, _ = P.decode_ref(pools[l], dec_turned[l], now)
            C.assert_decode_close(dec.out[l].cpu().numpy(), want)

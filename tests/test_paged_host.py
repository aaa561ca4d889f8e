"""The paged cache's and the log probabilities' entry points without a GPU: every bad
call is refused on the host before any CUDA work, and the workspace grows with the call."""
import ctypes
import math

import pytest
import torch

FAKE, MIS = 1 << 20, (1 << 20) + 8  # never dereferenced


def _desc(lib, **over):
    a = dict(batch=3, n_kv_heads=2, head_dim=128, page_size=16, n_pages=40, max_pages=8,
             dtype=lib.BF16, page_stride=0, head_stride=0, row_stride=0)
    a.update(over)
    return lib.PagedDesc(**a)


BAD_DESCS = [
    dict(batch=0), dict(n_kv_heads=0), dict(head_dim=96), dict(page_size=0), dict(page_size=24),
    dict(page_size=2048), dict(n_pages=0), dict(max_pages=0), dict(dtype=2),
    dict(max_pages=1 << 28), dict(max_pages=1 << 27),              # rows past int32
    dict(batch=(1 << 16) + 1), dict(batch=1 << 16, n_kv_heads=257),
    dict(page_stride=-4096, head_stride=2048, row_stride=128),
    dict(page_stride=4096, head_stride=2048, row_stride=132),      # not 16 bytes
    dict(page_stride=4096, head_stride=2048, row_stride=64),       # rows overlap
    dict(page_stride=4096, head_stride=1920, row_stride=128),      # heads overlap
    dict(page_stride=2048, head_stride=2048, row_stride=128),      # pages overlap
    dict(page_stride=0, head_stride=2048, row_stride=128),
]


def _append(lib, desc=None, rope=None, n=6, starts=None, hq=4, q=FAKE, qs=(512, 512, 128), q_out=FAKE * 2,
            os=(1024, 512, 128), k=FAKE, ks=(512, 256, 128), v=FAKE, vs=(512, 256, 128), pos=FAKE,
            kp=FAKE, vp=FAKE, table=FAKE, lens=FAKE):
    st = lambda s: ctypes.byref(lib.TokenStrides(*s)) if s is not None else None  # noqa: E731
    d = ctypes.byref(desc if desc is not None else _desc(lib))
    return lib._lib.ripple_paged_append(d, rope, n, starts, hq, q, st(qs), q_out, st(os), k, st(ks),
                                        v, st(vs), pos, kp, vp, table, lens, None, None)


def _rope(lib, rot=128, inter=0, freq=None, null=False):
    f = freq if freq is not None else [0.5] * 64
    arr = (ctypes.c_double * len(f))(*f)
    d = lib.RopeDesc(rot, inter, None if null else arr)
    d._arr = arr
    return ctypes.byref(d)


def test_append_refuses_bad_arguments(lib):
    E = lib.EINVAL
    for over in BAD_DESCS:
        assert _append(lib, desc=_desc(lib, **over)) == E, over
    assert _append(lib, n=-1) == E
    assert _append(lib, n=7) == E            # not a multiple of the batch
    assert _append(lib, q=None) == E         # q_out alone
    assert _append(lib, q_out=None) == E
    assert _append(lib, hq=0) == E
    for key in ("k", "v", "kp", "vp", "table", "lens"):
        assert _append(lib, **{key: None}) == E, key
    for key in ("q", "q_out", "k", "v", "kp", "vp"):
        assert _append(lib, **{key: MIS}) == E, key
    for key in ("qs", "os", "ks", "vs"):
        assert _append(lib, **{key: None}) == E, key
        assert _append(lib, **{key: (512, 260, 128)}) == E, key  # not 16 bytes
        assert _append(lib, **{key: (-512, 256, 128)}) == E, key
    assert _append(lib, os=(512, 512, 128)) == E     # two tokens of a sequence, four heads: overlap
    assert _append(lib, os=(1024, 512, 64)) == E
    assert _append(lib, q_out=FAKE, os=(2048, 512, 128)) == E  # in place with other strides
    for rope in (_rope(lib, rot=8), _rope(lib, rot=144, freq=[0.1] * 72), _rope(lib, rot=40),
                 _rope(lib, inter=2), _rope(lib, null=True), _rope(lib, freq=[math.nan] * 64),
                 _rope(lib, freq=[0.1] * 63 + [1e9]), _rope(lib, freq=[math.inf] * 64)):
        assert _append(lib, rope=rope) == E
    assert _append(lib, rope=_rope(lib, rot=128), desc=_desc(lib, head_dim=64)) == E
    # nothing to do: no launch, whatever the pointers
    assert _append(lib, n=0, q=None, q_out=None, k=None, v=None) == lib.OK
    assert _append(lib, n=0, rope=_rope(lib, rot=8)) == E


def _decode(lib, desc=None, hq=8, scale=0.0, q=FAKE, qs=(1024, 0, 128), kp=FAKE, vp=FAKE, table=FAKE,
            lens=FAKE, out=FAKE, ws=FAKE, wsb=1 << 30):
    d = ctypes.byref(desc if desc is not None else _desc(lib))
    s = ctypes.byref(lib.TokenStrides(*qs)) if qs is not None else None
    return lib._lib.ripple_paged_decode_attn(d, hq, scale, q, s, kp, vp, table, lens, out, None, ws,
                                             wsb, None, None)


def test_decode_refuses_bad_arguments(lib):
    E = lib.EINVAL
    for over in BAD_DESCS:
        assert _decode(lib, desc=_desc(lib, **over)) == E, over
    for hq in (0, 7, 34):  # none, not a multiple, 17 a group
        assert _decode(lib, hq=hq) == E
    for scale in (-1.0, math.inf, math.nan):
        assert _decode(lib, scale=scale) == E
    for key in ("q", "kp", "vp", "table", "lens", "out", "ws"):
        assert _decode(lib, **{key: None}) == E, key
    for key in ("q", "kp", "vp", "out", "ws"):
        assert _decode(lib, **{key: MIS}) == E, key
    assert _decode(lib, ws=FAKE + 16) == E
    for qs in ((1020, 0, 128), (1024, 0, 130), (-8, 0, 128)):
        assert _decode(lib, qs=qs) == E
    n = ctypes.c_size_t()
    assert lib._lib.ripple_paged_decode_workspace_bytes(ctypes.byref(_desc(lib)), 8,
                                                        ctypes.byref(n)) == lib.OK
    assert _decode(lib, wsb=n.value - 1) == lib.EWORKSPACE
    assert lib._lib.ripple_paged_decode_workspace_bytes(ctypes.byref(_desc(lib)), 34,
                                                        ctypes.byref(n)) == E


def test_words_are_aligned(lib):
    for key in ("pos", "table", "lens", "starts"):
        assert _append(lib, **{key: FAKE + 2}) == lib.EINVAL, key
    for key in ("table", "lens"):
        assert _decode(lib, **{key: FAKE + 2}) == lib.EINVAL, key


def test_decode_workspace_grows_with_the_call(lib):
    def need(hq=8, **over):
        n = ctypes.c_size_t()
        assert lib._lib.ripple_paged_decode_workspace_bytes(ctypes.byref(_desc(lib, **over)), hq,
                                                            ctypes.byref(n)) == lib.OK
        return n.value

    for sizes in ([need(batch=b) for b in range(1, 400)],
                  [need(max_pages=m) for m in range(1, 3000, 7)],
                  [need(hq=2 * g) for g in range(1, 17)],
                  [need(hq=8 * h, n_kv_heads=h) for h in range(1, 40)]):
        assert sizes == sorted(sizes)


def _logprobs(lib, n=4, vocab=100, stride=100, dtype=0, scale=1.0, top=2, logits=FAKE, tokens=FAKE,
              lp=FAKE, ent=None, lse=None, idx=FAKE, tlp=FAKE):
    return lib._lib.ripple_token_logprobs(n, vocab, stride, dtype, scale, top, logits, tokens, lp,
                                          ent, lse, idx, tlp, None, None)


def test_logprobs_refuses_bad_arguments(lib):
    E = lib.EINVAL
    for n in (-1, (1 << 27) + 1):
        assert _logprobs(lib, n=n) == E
    for vocab in (0, -5, (1 << 30) + 1):
        assert _logprobs(lib, vocab=vocab) == E
    assert _logprobs(lib, stride=-1) == E
    assert _logprobs(lib, dtype=2) == E
    for scale in (-1.0, math.inf, math.nan):
        assert _logprobs(lib, scale=scale) == E
    for top in (-1, 33):
        assert _logprobs(lib, top=top) == E
    assert _logprobs(lib, vocab=3, top=4) == E
    assert _logprobs(lib, logits=None) == E
    assert _logprobs(lib, tokens=None) == E          # logprob_out alone
    assert _logprobs(lib, lp=None) == E
    assert _logprobs(lib, idx=None) == E
    assert _logprobs(lib, top=0) == E                # top_idx_out without alternatives
    assert _logprobs(lib, top=0, idx=None) == E
    for key in ("logits", "tokens", "lp", "ent", "lse", "idx", "tlp"):
        assert _logprobs(lib, **{key: FAKE + 2}) == E, key
    assert _logprobs(lib, dtype=lib.BF16, logits=FAKE + 1) == E
    assert _logprobs(lib, n=0, logits=None, tokens=None, lp=None, idx=None, tlp=None) == lib.OK


def test_binding_refuses_host_tensors_and_wrong_shapes(lib):
    z = torch.zeros
    pages = z(4, 2, 16, 128, dtype=torch.bfloat16)
    table = z(3, 2, dtype=torch.int32)
    for k, v, t in [(pages, pages[:, :, :, :64], table), (pages[0], pages[0], table),
                    (pages, pages.float(), table), (pages, pages, table.long()),
                    (pages, pages, table[0]), (pages.transpose(2, 3), pages.transpose(2, 3), table),
                    (pages, pages, table)]:  # the last: on the host
        with pytest.raises(ValueError):
            lib.PagedCache(k, v, t)
    logits, tok, out = z(3, 50), z(3, dtype=torch.int32), z(3)
    for kw in (dict(tokens=tok), dict(tokens=tok.long(), logprob_out=out), dict(logprob_out=out),
               dict(entropy_out=z(4)), dict(top_logprob=z(3, 2)),
               dict(top_idx=z(3, 2, dtype=torch.int32), top_logprob=z(3, 3)),
               dict(top_idx=z(3, 2)), dict(tokens=tok, logprob_out=out)):  # the last: on the host
        with pytest.raises(ValueError):
            lib.ripple_token_logprobs(logits, **kw)
    with pytest.raises(ValueError):
        lib.ripple_token_logprobs(logits.t(), entropy_out=z(50))

"""The 8-bit pages', the drafts' and the kept rows' entry points without a GPU: every bad call is
refused on the host before any CUDA work, and the workspaces grow with the call."""
import ctypes
import math

import pytest
import torch

from tests.test_paged_host import BAD_DESCS, FAKE, MIS, _rope

FAR = 1 << 32


def _desc(lib, **over):
    a = dict(batch=3, n_kv_heads=2, head_dim=128, page_size=16, n_pages=40, max_pages=8,
             dtype=lib.BF16, page_stride=0, head_stride=0, row_stride=0)
    a.update(over)
    return lib.PagedDesc(**a)


def _scales(lib, k=FAR, v=FAR * 2, strides=(0, 0, 0)):
    return lib.PagedScales(k, v, *strides)


BAD_SCALES = [dict(k=None), dict(v=None), dict(strides=(-32, 16, 1)), dict(strides=(32, 15, 1)),
              dict(strides=(16, 16, 1)), dict(strides=(32, 16, 0)), dict(strides=(1 << 50, 16, 1))]
# of 8-bit pages: strides in bytes, multiples of 16
BAD8 = [d for d in BAD_DESCS if d.get("row_stride") != 132] + [
    dict(page_stride=4096, head_stride=2048, row_stride=136)]


def _st(lib, s):
    return ctypes.byref(lib.TokenStrides(*s)) if s is not None else None


def _append8(lib, desc=None, scales=(), rope=None, n=6, starts=None, hq=4, q=FAKE, qs=(512, 512, 128),
             q_out=FAKE * 2, os=(1024, 512, 128), k=FAKE, ks=(512, 256, 128), v=FAKE, vs=(512, 256, 128),
             pos=FAKE, kp=FAKE * 4, vp=FAKE * 8, table=FAKE, lens=FAKE):
    st = lambda s: _st(lib, s)  # noqa: E731
    d = ctypes.byref(desc if desc is not None else _desc(lib))
    s = None if scales is None else ctypes.byref(_scales(lib, **dict(scales)))
    return lib._lib.ripple_paged_append_q8(d, s, rope, n, starts, hq, q, st(qs), q_out, st(os), k,
                                           st(ks), v, st(vs), pos, kp, vp, table, lens, None, None)


def test_append_refuses_bad_arguments(lib):
    E = lib.EINVAL
    assert _append8(lib, scales=None) == E
    for s in BAD_SCALES:
        assert _append8(lib, scales=s) == E, s
    for over in BAD8:
        assert _append8(lib, desc=_desc(lib, **over)) == E, over
    for key in ("k", "v", "kp", "vp", "table", "lens", "q", "q_out"):
        assert _append8(lib, **{key: None}) == E, key
    for key in ("q", "q_out", "k", "v", "kp", "vp"):
        assert _append8(lib, **{key: MIS}) == E, key
    for key in ("pos", "table", "lens", "starts"):
        assert _append8(lib, **{key: FAKE + 2}) == E, key
    assert _append8(lib, n=-1) == E and _append8(lib, n=7) == E
    assert _append8(lib, rope=_rope(lib, freq=[math.nan] * 64)) == E
    pool = 40 * 2 * 16 * 128  # bytes of the codes
    # pools, scales and both among one another
    assert _append8(lib, kp=FAKE * 4, vp=FAKE * 4 + pool - 16) == E
    assert _append8(lib, scales=dict(k=FAR, v=FAR + 40 * 2 * 16 - 1)) == E
    for p in (FAKE * 4, FAKE * 8):
        for key in ("k", "v"):
            assert _append8(lib, scales={key: p + pool - 1}) == E
            assert _append8(lib, scales={key: p}) == E
    # nothing to do: no launch, whatever the pointers
    assert _append8(lib, n=0, q=None, q_out=None, k=None, v=None) == lib.OK
    assert _append8(lib, n=0, scales=BAD_SCALES[0]) == E


def _decode8(lib, desc=None, scales=(), hq=8, scale=0.0, q=FAKE, qs=(1024, 0, 128), kp=FAKE, vp=FAKE,
             table=FAKE, lens=FAKE, out=FAKE, ws=FAKE, wsb=1 << 30):
    d = ctypes.byref(desc if desc is not None else _desc(lib))
    s = None if scales is None else ctypes.byref(_scales(lib, **dict(scales)))
    return lib._lib.ripple_paged_decode_attn_q8(d, s, hq, scale, q, _st(lib, qs), kp, vp, table, lens,
                                                out, None, ws, wsb, None, None)


def test_decode_refuses_bad_arguments(lib):
    E = lib.EINVAL
    assert _decode8(lib, scales=None) == E
    for s in BAD_SCALES:
        assert _decode8(lib, scales=s) == E, s
    for over in BAD8:
        assert _decode8(lib, desc=_desc(lib, **over)) == E, over
    for hq in (0, 7, 34):
        assert _decode8(lib, hq=hq) == E
    for scale in (-1.0, math.inf, math.nan):
        assert _decode8(lib, scale=scale) == E
    for key in ("q", "kp", "vp", "table", "lens", "out", "ws"):
        assert _decode8(lib, **{key: None}) == E, key
    for key in ("q", "kp", "vp", "out", "ws"):
        assert _decode8(lib, **{key: MIS}) == E, key
    for key in ("table", "lens"):
        assert _decode8(lib, **{key: FAKE + 2}) == E, key
    for qs in ((1020, 0, 128), (1024, 0, 130), (-8, 0, 128)):
        assert _decode8(lib, qs=qs) == E
    n = ctypes.c_size_t()
    assert lib._lib.ripple_paged_decode_q8_workspace_bytes(ctypes.byref(_desc(lib)), 8,
                                                           ctypes.byref(n)) == lib.OK
    assert _decode8(lib, wsb=n.value - 1) == lib.EWORKSPACE
    assert lib._lib.ripple_paged_decode_q8_workspace_bytes(ctypes.byref(_desc(lib)), 34,
                                                           ctypes.byref(n)) == E
    assert lib._lib.ripple_paged_decode_q8_workspace_bytes(ctypes.byref(_desc(lib)), 8, None) == E


def test_decode_workspace_grows_with_the_call(lib):
    def need(hq=8, **over):
        n = ctypes.c_size_t()
        assert lib._lib.ripple_paged_decode_q8_workspace_bytes(ctypes.byref(_desc(lib, **over)), hq,
                                                               ctypes.byref(n)) == lib.OK
        return n.value

    for d in (64, 128):
        for sizes in ([need(batch=b, head_dim=d) for b in range(1, 400)],
                      [need(max_pages=m, head_dim=d) for m in range(1, 3000, 7)],
                      [need(hq=2 * g, head_dim=d, max_pages=3000) for g in range(1, 17)],
                      [need(hq=8 * h, n_kv_heads=h, head_dim=d) for h in range(1, 40)]):
            assert sizes == sorted(sizes)


def _tree(lib, desc=None, scales=None, n=12, starts=None, most=4, masks=FAKE, hq=8, scale=0.0, q=FAKE,
          qs=(4096, 1024, 128), kp=FAKE, vp=FAKE, table=FAKE, lens=FAKE, out=FAKE, lse=None, ws=FAKE,
          wsb=1 << 40, status=None):
    d = ctypes.byref(desc) if desc is not None else ctypes.byref(_desc(lib))
    s = None if scales is None else ctypes.byref(_scales(lib, **dict(scales)))
    return lib._lib.ripple_paged_tree_attn(d, s, n, starts, most, masks, hq, scale, q, _st(lib, qs), kp,
                                           vp, table, lens, out, lse, ws, wsb, status, None)


def _tree_bytes(lib, hq=8, most=4, scales=None, **over):
    n = ctypes.c_size_t()
    s = None if scales is None else ctypes.byref(_scales(lib, **dict(scales)))
    r = lib._lib.ripple_paged_tree_workspace_bytes(ctypes.byref(_desc(lib, **over)), s, hq, most,
                                                   ctypes.byref(n))
    return n.value if r == lib.OK else -r


def test_tree_refuses_bad_arguments(lib):
    E = lib.EINVAL
    for over in BAD_DESCS:
        assert _tree(lib, desc=_desc(lib, **over)) == E, over
    for over in BAD8:
        assert _tree(lib, desc=_desc(lib, **over), scales=()) == E, over
    for s in BAD_SCALES:
        assert _tree(lib, scales=s) == E, s
    for hq in (0, 7, 34):
        assert _tree(lib, hq=hq) == E
    for scale in (-1.0, math.inf, math.nan):
        assert _tree(lib, scale=scale) == E
    for most in (0, 3, 65):        # none, fewer than the batch has, too many
        assert _tree(lib, most=most) == E
    for n in (-3, 7):
        assert _tree(lib, n=n) == E
    for key in ("q", "kp", "vp", "table", "lens", "out", "ws", "qs"):
        assert _tree(lib, **{key: None}) == E, key
    for key in ("q", "kp", "vp", "out", "ws"):
        assert _tree(lib, **{key: MIS}) == E, key
    for key in ("table", "lens", "lse", "starts", "status"):
        assert _tree(lib, **{key: FAKE + 2}) == E, key
    assert _tree(lib, masks=FAKE + 4) == E
    assert _tree(lib, ws=FAKE + 16) == E
    for qs in ((4100, 1024, 128), (4096, 1028, 128), (4096, 1024, -128), (1 << 41, 1024, 128)):
        assert _tree(lib, qs=qs) == E
    assert _tree(lib, n=0, q=None, out=None) == lib.OK
    for dtype in (lib.BF16, lib.F32):
        for scales in (None, ()):
            need = _tree_bytes(lib, dtype=dtype, scales=scales)
            assert _tree(lib, desc=_desc(lib, dtype=dtype), scales=scales, wsb=need - 1) == lib.EWORKSPACE
    assert _tree_bytes(lib, hq=34) == -E and _tree_bytes(lib, most=65) == -E
    assert _tree_bytes(lib, scales=BAD_SCALES[0]) == -E


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("scales", [None, ()])
def test_tree_workspace_grows_with_the_call(lib, dtype, scales):
    need = lambda **a: _tree_bytes(lib, dtype=dtype, scales=scales, **a)  # noqa: E731
    for sizes in ([need(batch=b) for b in range(1, 400)],
                  [need(max_pages=m) for m in range(1, 3000, 7)],
                  [need(hq=2 * g, most=1) for g in range(1, 17)],
                  [need(hq=2 * g, most=33, max_pages=900) for g in range(1, 17)],
                  [need(most=m) for m in range(1, 65)],
                  [need(most=m, hq=32, max_pages=2000, batch=20) for m in range(1, 65)],
                  [need(hq=8 * h, n_kv_heads=h) for h in range(1, 40)]):
        assert sizes == sorted(sizes) and sizes[0] > 0


def _keep(lib, desc=None, scales=None, layers=2, ptrs=None, n=12, starts=None, most=4, kept=FAKE,
          lens=FAKE, lens_out=FAKE, null=None):
    d = ctypes.byref(desc) if desc is not None else ctypes.byref(_desc(lib))
    L = max(1, min(layers, 200))
    P = ctypes.c_void_p * L
    k, v, t = ptrs or ([FAKE * 4] * L, [FAKE * 8] * L, [FAKE] * L)
    arrays = [None if null == i else P(*x) for i, x in enumerate((k, v, t))]
    s = None
    if scales is not None:
        s = (lib.PagedScales * L)(*[_scales(lib, **dict(scales)) for _ in range(L)])
    return lib._lib.ripple_paged_keep_rows(d, s, layers, *arrays, n, starts, most, kept, lens, lens_out,
                                           None, None)


def test_keep_refuses_bad_arguments(lib):
    E = lib.EINVAL
    for over in BAD_DESCS:
        assert _keep(lib, desc=_desc(lib, **over)) == E, over
    for s in BAD_SCALES:
        assert _keep(lib, scales=s) == E, s
    for layers in (0, -1, 129):
        assert _keep(lib, layers=layers) == E
    for i in range(3):
        assert _keep(lib, null=i) == E
        for bad in ([None, FAKE * 4], [FAKE * 4, FAKE * 4 + 2]):
            ptrs = [[FAKE * 4] * 2, [FAKE * 8] * 2, [FAKE] * 2]
            ptrs[i] = bad
            assert _keep(lib, ptrs=ptrs) == E, (i, bad)
    assert _keep(lib, ptrs=[[FAKE * 4] * 2, [FAKE * 4 + 256] * 2, [FAKE] * 2]) == E  # pools overlap
    assert _keep(lib, n=-3) == E and _keep(lib, n=7) == E
    for most in (-1, 65):
        assert _keep(lib, most=most) == E
    assert _keep(lib, kept=None) == E
    for key in ("lens", "lens_out"):
        assert _keep(lib, **{key: None}) == E, key
    for key in ("lens", "lens_out", "kept", "starts"):
        assert _keep(lib, **{key: FAKE + 2}) == E, key
    # scales of other strides in another layer
    two = (lib.PagedScales * 2)(_scales(lib), _scales(lib, strides=(64, 32, 2)))
    P = ctypes.c_void_p * 2
    assert lib._lib.ripple_paged_keep_rows(
        ctypes.byref(_desc(lib)), two, 2, P(FAKE * 4, FAKE * 4), P(FAKE * 8, FAKE * 8), P(FAKE, FAKE),
        12, None, 4, FAKE, FAKE, FAKE, None, None) == E


def test_binding_refuses_host_tensors_and_wrong_shapes(lib):
    z = torch.zeros
    f8, e8 = torch.float8_e4m3fn, torch.float8_e8m0fnu
    pages = z(4, 2, 16, 128, dtype=torch.uint8).view(f8)
    s = z(4, 2, 16, dtype=torch.uint8).view(e8)
    table = z(3, 2, dtype=torch.int32)
    bf = z(4, 2, 16, 128, dtype=torch.bfloat16)
    for args, kw in [((pages, pages, table), {}), ((pages, pages, table), dict(k_scales=s)),
                     ((bf, bf, table), dict(k_scales=s, v_scales=s)),
                     ((bf, bf, table), dict(dtype=torch.float32)),
                     ((pages, pages, table), dict(k_scales=s, v_scales=s)),  # on the host
                     ((bf.half(), bf.half(), table), {})]:
        with pytest.raises((ValueError, KeyError)):
            lib.PagedCache(*args, **kw)

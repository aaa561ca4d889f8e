"""Appends whose outputs would be written over what other warps read are refused on the host;
views of one buffer that lie apart are not (what they give is tested on the GPU)."""
import ctypes
import itertools
import random

import pytest
import torch

from tests.test_paged_host import _desc, _rope

FAKE = 1 << 20  # never dereferenced: of bf16 elements
K, V, KP, VP = 1 << 24, 1 << 25, 1 << 30, 1 << 31


def _append(lib, q, qs, q_out, os, hq=4, n=6, starts=None, k=K, ks=(512, 256, 128), v=V,
            vs=(512, 256, 128), kp=KP, vp=VP, desc=None, rope=None):
    st = lambda s: ctypes.byref(lib.TokenStrides(*s)) if s is not None else None  # noqa: E731
    return lib._lib.ripple_paged_append(
        ctypes.byref(desc or _desc(lib)), rope, n, starts, hq, q, st(qs), q_out, st(os), k, st(ks),
        v, st(vs), FAKE, kp, vp, FAKE, FAKE, None, None)


def _accepts(lib, *args, **kw):
    """Without a GPU a call that is not refused ends at its launch."""
    if torch.cuda.is_available():
        pytest.skip("would launch on addresses that are none")
    return _append(lib, *args, **kw) == lib.ECUDA


# three sequences of two tokens, four query and two KV heads of 128: 1024 elements a token
DENSE = (1024, 512, 128)
FUSED = (2048, 1024, 128)


@pytest.mark.parametrize("shift", [8, 64, 128, 512, 520, 1024, 2048, 3000, -8, -128, -1024])
def test_queries_over_other_queries(lib, shift):
    assert _append(lib, FAKE, DENSE, FAKE + 2 * shift, DENSE) == lib.EINVAL


def test_queries_beside_other_queries(lib):
    end = 2 * (3 * 1024)
    for q_out in (FAKE + end, FAKE - end):
        assert _accepts(lib, FAKE, DENSE, q_out, DENSE)
    # in a token's row of one buffer
    assert _accepts(lib, FAKE, FUSED, FAKE + 2 * 512, FUSED)
    assert _append(lib, FAKE, FUSED, FAKE + 2 * 504, FUSED) == lib.EINVAL
    assert _append(lib, FAKE, FUSED, FAKE + 2 * 520, FUSED) == lib.EINVAL  # the next token's
    # with heads further apart than those it reads
    assert _accepts(lib, FAKE, (4096, 2048, 128), FAKE + 2 * 512, (4096, 2048, 256))
    assert _append(lib, FAKE, (4096, 2048, 128), FAKE + 2 * 504, (4096, 2048, 256)) == lib.EINVAL
    # in place
    assert _accepts(lib, FAKE, DENSE, FAKE, DENSE)


def test_queries_over_keys_and_values(lib):
    for over in (dict(k=FAKE, ks=FUSED), dict(v=FAKE, vs=FUSED)):
        name = "k" if "k" in over else "v"
        # q, then q_out over the first KV heads of the same token's row
        at = {name: FAKE + 2 * 512, name + "s": FUSED}
        for q_out in (FAKE + 2 * 512, FAKE + 2 * 640, FAKE + 2 * 256):
            assert _append(lib, 1 << 26, DENSE, q_out, FUSED, **at) == lib.EINVAL, (name, q_out)
        # in place, the keys among the queries' heads
        at = {name: FAKE + 2 * 256, name + "s": FUSED}
        assert _append(lib, FAKE, FUSED, FAKE, FUSED, **at) == lib.EINVAL
        at = {name: FAKE + 2 * 512, name + "s": FUSED}
        assert _accepts(lib, FAKE, FUSED, FAKE, FUSED, **at)


def test_ragged_tokens_count_whole(lib):
    # token 5 of six, the last
    assert _append(lib, FAKE, (0, 512, 128), FAKE + 2 * 5 * 512, (0, 512, 128), starts=FAKE) == lib.EINVAL
    assert _accepts(lib, FAKE, (0, 512, 128), FAKE + 2 * 6 * 512, (0, 512, 128), starts=FAKE)


def test_pools_over_one_another(lib):
    # dense pools of 40 pages of 2 x 16 rows of 128
    page = 2 * 16 * 128
    for vp in (KP, KP + 2 * 128, KP - 2 * 39 * page, KP + 2 * 39 * page):
        assert _append(lib, None, None, None, None, vp=vp) == lib.EINVAL, vp - KP
    assert _accepts(lib, None, None, None, None, vp=KP + 2 * 40 * page)
    # a page of both in one allocation, and heads of both in a row
    both = _desc(lib, page_stride=2 * page, head_stride=16 * 128, row_stride=128)
    assert _accepts(lib, None, None, None, None, vp=KP + 2 * page, desc=both)
    assert _append(lib, None, None, None, None, vp=KP + 2 * page - 16, desc=both) == lib.EINVAL
    rows = _desc(lib, page_stride=16 * 512, head_stride=128, row_stride=512)
    assert _accepts(lib, None, None, None, None, vp=KP + 2 * 256, desc=rows)
    assert _append(lib, None, None, None, None, vp=KP + 2 * 128, desc=rows) == lib.EINVAL


def test_spans_that_no_tensor_has(lib):
    big = 1 << 40
    assert _append(lib, FAKE, (512, big, 128), 1 << 26, (1 << 21, 512, 128), n=3 << 10) == lib.EINVAL
    assert _append(lib, FAKE, DENSE, 1 << 26, (128, big, 0), hq=1, n=3 << 10) == lib.EINVAL


def test_against_every_place(lib):
    """Random small layouts of q and q_out against the places themselves."""
    if torch.cuda.is_available():
        pytest.skip("would launch on addresses that are none")
    rng = random.Random(5)
    B, m, hq, d = 3, 2, 2, 64
    desc = _desc(lib, head_dim=d)
    said = set()
    for _ in range(4000):
        def strides():
            order = [B, m, hq]
            s, at = [0, 0, 0], d
            for i in rng.sample(range(3), 3):  # each dimension past those within it
                s[i] = at + rng.choice([0, 0, 8, 64, 128])
                at = s[i] * order[i] + rng.choice([0, 0, 64])
            return s
        qs = strides()
        os = list(qs) if rng.random() < 0.6 else strides()
        shift = rng.randrange(-300, 300) * 8
        at = lambda s: [b * s[0] + i * s[1] + h * s[2]  # noqa: E731
                        for b, i, h in itertools.product(range(B), range(m), range(hq))]
        clash = any(abs(x - (y + shift)) < d for x in at(qs) for y in at(os))
        clash = clash and not (shift == 0 and qs == os)
        status = _append(lib, FAKE, qs, FAKE + 2 * shift, os, hq=hq, desc=desc, ks=(256, 128, 64),
                         vs=(256, 128, 64))
        if clash or (shift == 0 and qs != os):
            assert status == lib.EINVAL, (qs, os, shift)
        elif qs == os:  # other layouts may be refused where only their spans meet
            assert status == lib.ECUDA, (qs, os, shift)
        said.add((clash, qs == os, status))
    assert {(True, True, lib.EINVAL), (False, True, lib.ECUDA), (True, False, lib.EINVAL),
            (False, False, lib.ECUDA)} <= said


def test_what_else_is_refused_of_an_accepted_call(lib):
    good = dict(q=FAKE, qs=DENSE, q_out=1 << 26, os=DENSE)
    assert _accepts(lib, **good)
    assert _accepts(lib, **good, rope=_rope(lib))
    for over in [dict(n=7), dict(hq=0), dict(k=None), dict(v=K + 8), dict(kp=KP + 8), dict(vp=None),
                 dict(qs=(1024, 516, 128)), dict(os=(1024, -512, 128)), dict(os=(512, 512, 128)),
                 dict(os=(1024, 512, 64)), dict(rope=_rope(lib, rot=40)),
                 dict(desc=_desc(lib, page_size=24))]:
        assert _append(lib, **dict(good, **over)) == lib.EINVAL, over

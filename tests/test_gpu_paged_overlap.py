"""ripple_paged_append on tensors that share a buffer: queries rotated into heads beside
those of the same token give what separate tensors give, and overlapping ones are refused
before any launch."""
import pytest
import torch

from tests import paged_common as P

pytestmark = pytest.mark.gpu
DEV = "cuda"
HQ, H, D = 4, 2, 64
INV = [100.0 ** (-2.0 * j / D) for j in range(D // 2)]


def _views(wide, ragged):
    """q, k, v and room for q's rotation in a token's row; every second head for the last."""
    q, k, v, rest = wide.split([HQ, H, H, 2 * HQ], dim=-2)
    return q, k, v, rest[..., ::2, :]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ragged", [False, True])
def test_queries_beside_those_of_the_same_row(lib, ragged, dtype):
    rows, new = [40, 3, 17], [3, 3, 3]
    shape = (9,) if ragged else (3, 3)
    wide = P.randn((*shape, 4 * HQ, D), dtype, 1)
    q, k, v, q_out = _views(wide, ragged)
    kw = dict(seq_starts=P.i32([0, 3, 6, 9])) if ragged else {}
    pools = [P.Pool(lib, rows, H, D, 8, dtype, 2) for _ in range(2)]
    apart = torch.zeros_like(q, memory_format=torch.contiguous_format)
    lib.ripple_paged_append(pools[0].cache, P.i32(rows), k.clone(), v.clone(), rope=lib.Rope(INV),
                            q=q.clone(), q_out=apart, **kw)
    before = wide.clone()
    lib.ripple_paged_append(pools[1].cache, P.i32(rows), k, v, rope=lib.Rope(INV), q=q, q_out=q_out,
                            **kw)
    torch.cuda.synchronize()
    assert torch.equal(q_out, apart)
    for x, y in ((pools[0].k, pools[1].k), (pools[0].v, pools[1].v)):
        assert torch.equal(x, y)
    _views(before, ragged)[3].copy_(apart)
    assert torch.equal(wide, before)  # and nothing else in the buffer


def test_overlapping_tensors_are_refused(lib):
    wide = P.randn((6, 4 * HQ, D), "bf16", 3)
    q, k, v = wide[:, :HQ], wide[:, HQ:HQ + H], wide[:, HQ + H:HQ + 2 * H]
    rows = [4] * 6
    pool = P.Pool(lib, rows, H, D, 8, "bf16", 4)
    launches = lib.ripple_kernel_launches()
    for q_out in (wide[:, 1:1 + HQ], wide[:, HQ - 1:2 * HQ - 1], wide[:, HQ:2 * HQ],
                  wide[:, HQ + H:2 * HQ + H], wide.flatten()[8:8 + 6 * HQ * D].view(6, HQ, D)):
        with pytest.raises(lib.RippleError) as e:
            lib.ripple_paged_append(pool.cache, P.i32(rows), k, v, q=q, q_out=q_out)
        assert e.value.status == lib.EINVAL
    same = lib.PagedCache(pool.k, pool.k, pool.table)
    with pytest.raises(lib.RippleError) as e:
        lib.ripple_paged_append(same, P.i32(rows), k, v)
    assert e.value.status == lib.EINVAL
    assert lib.ripple_kernel_launches() == launches
    # reading keys as values is no harm
    out = torch.empty(6, HQ, D, device=DEV)
    ws = torch.empty(lib.ripple_paged_decode_workspace_bytes(same, HQ), dtype=torch.uint8, device=DEV)
    lib.ripple_paged_decode_attn(same, q, P.i32(rows), out, ws)
    torch.cuda.synchronize()
    assert torch.isfinite(out).all()

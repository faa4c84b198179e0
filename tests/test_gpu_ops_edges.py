"""Calls at the edges of what the operators around a cache take."""
import pytest
import torch

import paper_2604_15750_b200 as dc

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, BF16, E4M3 = torch.float32, torch.bfloat16, torch.float8_e4m3fn


@pytest.mark.parametrize("held", [E4M3, BF16])
def test_calls_of_nothing(held):
    """No sequences, no rows, no layers: nothing is done, as qk_norm_rope of no rows does nothing."""
    c = dc.KvCache.empty(2, 3, 2, 64, 128, held, DEV)
    for layers, batch, rows in ((1, 0, 4), (2, 3, 0), (0, 3, 4), (0, 0, 0)):
        x = torch.empty((layers, batch, rows, 2, 128), dtype=BF16, device=DEV)
        assert dc.cache_write(c, x, x, [5] * batch) is c
        assert dc.cache_read(c, x, x.clone(), [5] * batch, [0] * batch)[0] is x
        with pytest.raises(ValueError):
            dc.cache_write(c, x, x, [5] * (batch + 1))
    for batch, rows in ((0, 4), (3, 0), (0, 0)):
        q = torch.empty((batch, rows, 4, 128), dtype=BF16, device=DEV)
        mask = torch.empty((batch, rows, (rows + 31) // 32), dtype=torch.int32, device=DEV)
        for kw in (dict(), dict(mask=mask), dict(out=torch.empty_like(q))):
            assert dc.tree_attention(q, c, [9] * batch, [0] * batch, **kw).shape == q.shape
        assert dc.tree_attention_workspace(q, c, [9] * batch, [0] * batch) == 0
        with pytest.raises(ValueError):
            dc.tree_attention(q, c, [9] * batch, [0] * (batch + 1))
    assert not c.k.view(torch.uint8).any() and not c.v.view(torch.uint8).any()


@pytest.mark.parametrize("dtype,held,hd", [(BF16, E4M3, 128), (BF16, BF16, 128), (F32, F32, 64), (BF16, BF16, 96)])
@pytest.mark.parametrize("ctx,rows,group", [([500] * 4, [9] * 4, 1), ([1000, 20], [100, 3], 2), ([40000, 20], [9, 3], 2)])
def test_attention_in_the_place_of_the_queries(dtype, held, hd, ctx, rows, group):
    """out = q: units on their own, joined by a cluster and by a launch give what they give elsewhere."""
    g = torch.Generator().manual_seed(5)
    B, H, most = len(ctx), 2, max(rows) + 2
    if hd == 96:
        ctx = [min(x, 5000) for x in ctx]
    c = dc.KvCache.empty(1, B, H, (max(ctx) + most + 63) // 64 * 64, hd, held, DEV)
    x = torch.randn((B, c.max_ctx, H, hd), generator=g).to(dtype).to(DEV)
    dc.cache_write(c, x, x, [0] * B)
    q = torch.randn((B, most, H * group, hd), generator=g).to(dtype).to(DEV)
    mask = dc.tree_mask([[-1] + list(range(r - 1)) for r in rows], most).to(DEV)
    want = dc.tree_attention(q, c, ctx, rows, mask)
    got = q.clone()
    assert dc.tree_attention(got, c, ctx, rows, mask, out=got) is got
    for b, r in enumerate(rows):
        assert torch.equal(got[b, :r], want[b, :r]) and torch.equal(got[b, r:], q[b, r:])


@pytest.mark.parametrize("theta,hd", [(10.0, 256), (10.0, 128), (1e4, 256), (2.0, 96)])
def test_the_farthest_positions_keep_their_angles(theta, hd):
    """An angle of 2^31 x a frequency is 2^53 of its own roundings away from a turn only if the frequency is off by one of them:
    the tolerance has none beside it."""
    import ops_ref as ref
    g = torch.Generator().manual_seed(7)
    q, k = (torch.randn((500, 3, hd), generator=g) for _ in range(2))
    pos = torch.randint(2 ** 30, 2 ** 31 - 1, (500,), generator=g, dtype=torch.int32)
    outs = dc.qk_norm_rope(q.to(DEV), k.to(DEV), pos.to(DEV), eps=1e-6, rope_theta=theta)
    for got, x in zip(outs, (q, k)):
        want, size = ref.rope(x, pos, None, 1e-6, theta)
        over = (got.cpu().double() - want).abs() / ref.rope_tolerance(want, size, F32)
        assert (over <= 1).all(), float(over.max())

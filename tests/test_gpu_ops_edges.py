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

"""The bounded waits of the attention of drafted rows on the tensor cores, run out on purpose as in test_gpu_timeout.py: producers
that ask for fewer tiles than the others wait for.  The kernel comes back with NaN in the rows concerned and DC_ERR_TIMEOUT in the
status, and the next call is clean."""
import time

import pytest
import torch

import paper_2604_15750_b200 as dc
from paper_2604_15750_b200 import inputs
from paper_2604_15750_b200.binding import DC_ERR_TIMEOUT, DC_OPT_TEST_STALL_TREE, DC_OPT_WAIT_LIMIT_US

from parity import Case

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16, E4M3 = torch.bfloat16, torch.float8_e4m3fn
NO_TILE, FIRST_TILE, SECOND_STRETCH = 1, 2, 3


@pytest.fixture(scope="module")
def engine():
    eng = Case(inputs.Workload("wait_limit", 2, 256, 2, 2, 128, 512, 2048, "bf16", 2, 40, 64, 16, 32, 64, 31337)).make_engine()
    yield eng
    eng.close()


def _call(held, batch, heads, group, ctx, rows, masked):
    g = torch.Generator().manual_seed(3)
    most = max(rows) + 1
    c = dc.KvCache.empty(1, batch, heads, (max(ctx) + most + 63) // 64 * 64, 128, held, DEV)
    x = torch.randn((batch, c.max_ctx, heads, 128), generator=g).to(BF16).to(DEV)
    dc.cache_write(c, x, x, [0] * batch)
    q = torch.randn((batch, most, heads * group, 128), generator=g).to(BF16).to(DEV)
    mask = dc.tree_mask([[-1] + list(range(r - 1)) for r in rows], most).to(DEV) if masked else None
    status = torch.zeros(1, dtype=torch.int32, device=DEV)

    def run():
        out, _ = torch.full_like(q, 5.0), status.zero_()
        dc.tree_attention(q, c, ctx, rows, mask, out=out, status=status)
        torch.cuda.synchronize()
        return out, int(status)
    return run


# every sequence on its own (a unit for every place of the SMs, for 32, 64 and 128 lines); few units, whose stretches a cluster or a
# second launch joins, beside a sequence of one stretch
ALONE = [(8, 37, 1, [500] * 8, [8] * 8), (4, 37, 1, [500] * 4, [64] * 4), (4, 37, 1, [500] * 4, [128] * 4)]
JOINED = [(2, 1, 1, [1000, 20], [9, 3]), (2, 1, 2, [1000, 20], [128, 3]), (2, 1, 1, [40000, 20], [9, 3]), (2, 1, 4, [40000, 20], [64, 3])]


@pytest.mark.parametrize("held", [E4M3, BF16])
@pytest.mark.parametrize("how,call", [(h, c) for h in (NO_TILE, FIRST_TILE) for c in ALONE] +
                         [(h, c) for h in (NO_TILE, SECOND_STRETCH) for c in JOINED])
def test_waits_that_run_out(engine, held, how, call):
    batch, heads, group, ctx, rows = call
    run = _call(held, batch, heads, group, ctx, rows, masked=how != NO_TILE)
    ref, status = run()
    assert status == 0 and torch.isfinite(ref).all()
    try:
        engine.set_option(DC_OPT_WAIT_LIMIT_US, 20_000)
        engine.set_option(DC_OPT_TEST_STALL_TREE, how)
        t0 = time.perf_counter()
        out, status = run()
        took = time.perf_counter() - t0
    finally:
        engine.set_option(DC_OPT_TEST_STALL_TREE, 0)
        engine.set_option(DC_OPT_WAIT_LIMIT_US, 2_000_000)
    assert status == DC_ERR_TIMEOUT
    assert took < 1.5, took                               # 20 ms a wait, not the default 2 s
    for b, r in enumerate(rows):
        if how == SECOND_STRETCH and b == 1:
            assert torch.equal(out[b, :r], ref[b, :r])    # (it has no second stretch)
        else:
            assert torch.isnan(out[b, :r]).all()
        assert (out[b, r:] == 5).all()
    again, status = run()
    assert status == 0 and torch.equal(again, ref)

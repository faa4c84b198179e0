"""How dc_tree_attention splits calls, as its workspace shows it: on the host, without a GPU."""
import ctypes as C

import paper_2604_15750_b200 as dc
from paper_2604_15750_b200 import binding as b

L = dc.load_library()
A = 0x7F0000001000          # an aligned address that nothing follows


def workspace(ctx, rows, heads, max_ctx, batch=1, hkv=1, hd=128, held=b.DC_E4M3, dtype=b.DC_BF16, slots=None):
    scales = A if held == b.DC_E4M3 else None
    c = b.dc_cache(dtype=held, n_layers=1, max_batch=slots or batch, n_kv_heads=hkv, max_ctx=max_ctx, head_dim=hd, k=A, v=A, k_scale=scales, v_scale=scales)
    ints = lambda v: C.cast((C.c_int32 * batch)(*([v] * batch)), C.c_void_p)
    t = b.dc_tree_in(batch=batch, layer=0, dtype=dtype, n_q_heads=heads, max_rows=rows, scale=0.0, q=A, o=A, q_stride=(C.c_int64 * 3)(1, 1, 1),
                     o_stride=(C.c_int64 * 3)(1, 1, 1), ctx_len=ints(ctx), n_rows=ints(rows), mask=None)
    need = C.c_uint64()
    return L.dc_tree_attention_workspace(C.byref(c), C.byref(t), C.byref(need)), need.value


def test_no_stretch_over_an_8_bit_cache_is_longer_than_2_to_the_17_keys():
    """Its probabilities end 2^-27 below the largest of a stretch: 2^17 keys that are lost are 2^-10 of it at most.  More stretches than
    a cluster has CTAs want partial sums in a workspace, 8 + 4 x 128 bytes a line and stretch, however many units there are."""
    batch, hkv, keys = 8, 37, 1_310_720
    rc, need = workspace(keys - 1, 1, hkv, keys, batch, hkv)
    assert rc == 0 and need >= keys // 2 ** 17 * batch * hkv * (8 + 4 * 128)


def test_contexts_of_more_than_2_to_the_30_keys_are_refused():
    """Places of keys are 32-bit numbers, and those of the tiles behind the last one have to fit too."""
    most = 2 ** 31 - 64
    for hd, held, dtype in ((8, b.DC_E4M3, b.DC_BF16), (128, b.DC_E4M3, b.DC_BF16), (64, b.DC_F32, b.DC_F32)):
        for ctx in (most - 1, 2 ** 30):
            assert workspace(ctx, 1, 1, most, hd=hd, held=held, dtype=dtype)[0] == 3 and L.dc_last_error(None)
        rc, need = workspace(2 ** 30 - 1, 1, 1, most, hd=hd, held=held, dtype=dtype)
        assert rc == 0 and need > 0


def test_more_units_than_a_grid_has_are_refused_when_the_workspace_is_asked_for():
    """Not by the call alone, when its workspace has been made."""
    for rows, batch, hd, rc in ((256, 31, 256, 0), (256, 32, 256, 3)):
        assert workspace(10, rows, 128, 512, batch=batch, hd=hd)[0] == rc

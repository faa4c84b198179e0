"""What the operators around a cache refuse, before anything is launched: on the C entries with made-up addresses (never
followed), and on the binding with CPU tensors.  Runs without a GPU."""
import ctypes as C

import pytest
import torch

import paper_2604_15750_b200 as dc
from paper_2604_15750_b200 import binding as b

L = dc.load_library()
A = 0x7F0000001000          # an aligned address that nothing follows


def ints(*v):
    return C.cast((C.c_int32 * max(len(v), 1))(*v), C.c_void_p)


def cache(**kw):
    d = dict(dtype=b.DC_E4M3, n_layers=2, max_batch=4, n_kv_heads=2, max_ctx=128, head_dim=128, k=A, v=A, k_scale=A, v_scale=A)
    d.update(kw)
    return b.dc_cache(**d)


def rows(**kw):
    d = dict(batch=2, layer=0, n_layers=1, dtype=b.DC_BF16, k=A, v=A, k_stride=(C.c_int64 * 5)(0, 0, 256, 128, 1),
             v_stride=(C.c_int64 * 5)(0, 0, 256, 128, 1), pos=ints(0, 5), n=ints(0, 0))
    d.update(kw)
    return b.dc_cache_rows(**d)


def tree(**kw):
    d = dict(batch=2, layer=1, dtype=b.DC_BF16, n_q_heads=4, max_rows=16, scale=0.0, q=A, o=A, q_stride=(C.c_int64 * 3)(1, 1, 1),
             o_stride=(C.c_int64 * 3)(1, 1, 1), ctx_len=ints(10, 0), n_rows=ints(0, 0), mask=A)
    d.update(kw)
    return b.dc_tree_in(**d)


def qk(**kw):
    d = dict(dtype=b.DC_BF16, rows=0, n_q_heads=4, n_kv_heads=2, head_dim=128, eps=1e-6, rope_theta=1e4, q=A, k=A, pos=A, q_out=A, k_out=A)
    d.update(kw)
    return b.dc_qk_in(**d)


INVALID, SHAPE, UNSUPPORTED = 1, 2, 3
BAD_CACHES = [
    (dict(dtype=7), INVALID), (dict(n_layers=0), INVALID), (dict(max_batch=-1), INVALID), (dict(max_ctx=100), INVALID),
    (dict(head_dim=12), UNSUPPORTED), (dict(head_dim=264), UNSUPPORTED), (dict(head_dim=0), UNSUPPORTED), (dict(k=None), INVALID),
    (dict(v=None), INVALID), (dict(k_scale=None), INVALID), (dict(v_scale=None), INVALID), (dict(dtype=b.DC_BF16), INVALID),
]


@pytest.mark.parametrize("bad,code", BAD_CACHES)
def test_caches(bad, code):
    c, need = cache(**bad), C.c_uint64(7)
    assert L.dc_cache_write(C.byref(c), C.byref(rows()), None) == code
    assert L.dc_cache_read(C.byref(c), C.byref(rows()), None) == code
    assert L.dc_tree_attention(C.byref(c), C.byref(tree()), None) == code
    assert L.dc_tree_attention_workspace(C.byref(c), C.byref(tree()), C.byref(need)) == code and need.value == 7
    assert L.dc_last_error(None)


@pytest.mark.parametrize("bad,code", [
    (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(dtype=b.DC_E4M3), INVALID), (dict(batch=0), SHAPE), (dict(batch=5), SHAPE),
    (dict(layer=-1), SHAPE), (dict(layer=1, n_layers=2), SHAPE), (dict(n_layers=0), SHAPE), (dict(n_layers=2 ** 31 - 1, layer=1), SHAPE),
    (dict(pos=None), INVALID), (dict(n=None), INVALID), (dict(pos=ints(-1, 0)), SHAPE), (dict(n=ints(0, -1)), SHAPE),
    (dict(pos=ints(0, 100), n=ints(0, 29)), SHAPE), (dict(pos=ints(0, 2 ** 31 - 1), n=ints(0, 2 ** 31 - 1)), SHAPE), (dict(n=ints(129, 0)), SHAPE),
])
def test_rows(bad, code):
    for f in (L.dc_cache_write, L.dc_cache_read):
        assert f(C.byref(cache()), C.byref(rows(**bad)), None) == code
        assert L.dc_last_error(None)


def test_rows_of_another_type_than_a_plain_cache():
    c = cache(dtype=b.DC_F32, k_scale=None, v_scale=None)
    assert L.dc_cache_write(C.byref(c), C.byref(rows()), None) == UNSUPPORTED
    assert L.dc_tree_attention(C.byref(c), C.byref(tree()), None) == UNSUPPORTED
    c = cache(max_batch=64)
    assert L.dc_cache_write(C.byref(c), C.byref(rows(batch=33)), None) == SHAPE      # DC_MAX_BATCH


def test_null_arguments_and_nothing_to_do():
    assert L.dc_cache_write(None, C.byref(rows()), None) == INVALID
    assert L.dc_cache_write(C.byref(cache()), None, None) == INVALID
    assert L.dc_tree_attention(C.byref(cache()), None, None) == INVALID
    assert L.dc_tree_attention_workspace(C.byref(cache()), C.byref(tree()), None) == INVALID
    assert L.dc_qk_norm_rope(None, None) == INVALID
    # without rows nothing is launched
    assert L.dc_cache_write(C.byref(cache()), C.byref(rows()), None) == 0
    assert L.dc_cache_read(C.byref(cache()), C.byref(rows()), None) == 0
    assert L.dc_tree_attention(C.byref(cache()), C.byref(tree()), None) == 0
    assert L.dc_qk_norm_rope(C.byref(qk()), None) == 0
    assert L.dc_qk_norm_rope(C.byref(qk(rows=3, n_q_heads=0, n_kv_heads=0)), None) == 0


@pytest.mark.parametrize("bad,code", [
    (dict(dtype=b.DC_E4M3), INVALID), (dict(batch=0), SHAPE), (dict(batch=5), SHAPE), (dict(layer=2), SHAPE), (dict(layer=-1), SHAPE),
    (dict(n_q_heads=3), INVALID), (dict(n_q_heads=0), INVALID), (dict(n_q_heads=4098, n_rows=ints(1, 0)), UNSUPPORTED),
    (dict(n_q_heads=1 << 18, max_rows=1, n_rows=ints(1, 0)), UNSUPPORTED), (dict(max_rows=0), SHAPE), (dict(max_rows=257), SHAPE),
    (dict(scale=-1.0), INVALID), (dict(scale=float("nan")), INVALID), (dict(scale=float("inf")), INVALID), (dict(scale=1e31), INVALID), (dict(ctx_len=None), INVALID),
    (dict(n_rows=None), INVALID), (dict(ctx_len=ints(-1, 0)), SHAPE), (dict(n_rows=ints(0, 17)), SHAPE), (dict(n_rows=ints(-1, 1)), SHAPE),
    (dict(ctx_len=ints(120, 0), n_rows=ints(9, 0)), SHAPE), (dict(ctx_len=ints(2 ** 31 - 1, 0), n_rows=ints(16, 0)), SHAPE),
    (dict(q=None), INVALID), (dict(o=None), INVALID),
])
def test_trees(bad, code):
    assert L.dc_tree_attention(C.byref(cache()), C.byref(tree(**bad)), None) == code
    assert L.dc_last_error(None)


def test_a_workspace_that_is_missing_too_small_or_off_its_boundary():
    c = cache(max_ctx=64 * 1024)
    t = dict(batch=1, ctx_len=ints(60000), n_rows=ints(16))
    need = C.c_uint64()
    assert L.dc_tree_attention_workspace(C.byref(c), C.byref(tree(**t)), C.byref(need)) == 0 and need.value > 0
    for bad in (dict(), dict(workspace=A, workspace_bytes=need.value - 1), dict(workspace=A + 8, workspace_bytes=need.value)):
        assert L.dc_tree_attention(C.byref(c), C.byref(tree(**t, **bad)), None) == INVALID
        assert b"workspace" in L.dc_last_error(None)


@pytest.mark.parametrize("bad,code", [
    (dict(dtype=2), INVALID), (dict(rows=-1), INVALID), (dict(n_q_heads=-1), INVALID), (dict(head_dim=3), UNSUPPORTED),
    (dict(head_dim=258), UNSUPPORTED), (dict(head_dim=0), UNSUPPORTED), (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID),
    (dict(rope_theta=0.0), INVALID), (dict(rope_theta=float("inf")), INVALID), (dict(rows=1, pos=None), INVALID), (dict(rows=1, q=None), INVALID),
    (dict(rows=1, k_out=None), INVALID), (dict(n_kv_heads=40000), UNSUPPORTED),
])
def test_heads(bad, code):
    assert L.dc_qk_norm_rope(C.byref(qk(**bad)), None) == code
    assert L.dc_last_error(None)


# ---- masks of trees (host) ------------------------------------------------------------------------------
def test_tree_mask():
    parents = [[-1, 0, 0, 1, -1, 4] + list(range(5, 70)), [], [-1]]
    m = dc.tree_mask(parents)
    assert m.shape == (3, 71, 3) and m.dtype == torch.int32
    for s, p in enumerate(parents):
        seen = []
        for i, q in enumerate(p):
            seen.append((seen[q] if q >= 0 else set()) | {i})
            assert {j for j in range(96) if (int(m[s, i, j // 32]) >> (j % 32)) & 1} == seen[i]
        assert not m[s, len(p):].any()
    assert dc.tree_mask([[-1, 0]], rows=40).shape == (1, 40, 2)


@pytest.mark.parametrize("p", [[0], [-1, 1], [-1, 2, 0], [-2], [-1] * 257])
def test_masks_of_what_is_no_tree(p):
    with pytest.raises(dc.DepCapError):
        dc.tree_mask([p])
    with pytest.raises(ValueError):
        dc.tree_mask([[-1, 0]], rows=1)


def test_the_packed_structures_are_those_of_the_header():
    from paper_2604_15750_b200 import ops
    assert [x.size for x in (ops._CACHE, ops._ROWS, ops._QK, ops._TREE)] == \
        [C.sizeof(x) for x in (b.dc_cache, b.dc_cache_rows, b.dc_qk_in, b.dc_tree_in)] == [56, 128, 152, 136]
    for packed, t in ((ops._CACHE, b.dc_cache), (ops._ROWS, b.dc_cache_rows), (ops._QK, b.dc_qk_in), (ops._TREE, b.dc_tree_in)):
        flat, at = [], 0
        for name, kind in t._fields_:
            flat += [(name, i) for i in range(kind._length_)] if hasattr(kind, "_length_") else [(name, None)]
        s = t.from_buffer_copy(packed.pack(*range(1, len(flat) + 1)))
        for i, (name, j) in enumerate(flat):
            v = getattr(s, name)
            assert (v if j is None else v[j]) == i + 1, name


# ---- the binding ------------------------------------------------------------------------------------------
def _kv(dtype=torch.bfloat16, hd=128):
    return torch.zeros((1, 2, 2, 64, hd), dtype=dtype), torch.zeros((1, 2, 2, hd, 64), dtype=dtype)


def test_the_binding_refuses():
    k, v = _kv()
    for bad in [(k, k), (k[0], v[0]), (k, v.float()), (k, v, torch.zeros(1, 2, 2, 64)), _kv(torch.float8_e4m3fn), (k.transpose(0, 1), v),
                (*_kv(torch.float8_e4m3fn), torch.zeros(1, 2, 2, 64), torch.zeros(1, 2, 2, 32)), (k[..., ::2], v[..., ::2, :])]:
        with pytest.raises(ValueError):
            dc.KvCache(*bad)
    with pytest.raises(TypeError):
        dc.KvCache(*_kv(torch.float16))
    c = dc.KvCache(k, v)
    x = torch.zeros((2, 3, 2, 128), dtype=torch.bfloat16)
    with pytest.raises(RuntimeError, match="no CPU path"):
        dc.cache_write(c, x, x, [0, 0])
    for bad in [(x, x[:, :2], [0, 0]), (x, x.float(), [0, 0]), (x, x, [0]), (x, x, [0, 0], [1]), (x, x, [0, 0], [4, 0]),
                (x[..., :64], x[..., :64], [0, 0]), (x[:, :, :1], x[:, :, :1], [0, 0]), (x, x, [0, 2 ** 40])]:
        with pytest.raises(ValueError):
            dc.cache_write(c, *bad)
    with pytest.raises(ValueError, match="expanded"):
        dc.cache_read(c, x[:, :1].expand(2, 3, 2, 128), x, [0, 0])
    q = torch.zeros((2, 3, 4, 128), dtype=torch.bfloat16)
    with pytest.raises(RuntimeError, match="no CPU path"):
        dc.tree_attention(q, c, [0, 0], [3, 3])
    for kw in [dict(mask=torch.zeros((2, 3, 2), dtype=torch.int32)), dict(mask=torch.zeros((2, 3, 1))), dict(out=q[:, :2]), dict(out=q.float()),
               dict(scale=0.0), dict(scale=-1.0), dict(status=torch.zeros(2, dtype=torch.int32)),
               dict(workspace=torch.zeros(1, dtype=torch.uint8).expand(1 << 20)), dict(out=q[:, :1].expand(2, 3, 4, 128))]:
        with pytest.raises(ValueError):
            dc.tree_attention(q, c, [0, 0], [3, 3], **kw)
    for bad in [(q[..., :64], c, [0, 0], [3, 3]), (q[0], c, [0, 0], [3, 3]), (q, c, [0], [3, 3]), (q.transpose(2, 3).contiguous().transpose(2, 3), c, [0, 0], [3, 3])]:
        with pytest.raises(ValueError):
            dc.tree_attention(*bad)
    h = torch.zeros((3, 4, 128), dtype=torch.bfloat16)
    pos = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(RuntimeError, match="no CPU path"):
        dc.qk_norm_rope(h, h, pos)
    for args, kw in [((h, h[:2], pos), {}), ((h, h.float(), pos), {}), ((h, h, pos.long()), {}), ((h, h, pos[:2]), {}), ((h[..., ::2], h[..., ::2], pos), {}),
                     ((h, h, pos), dict(q_gain=torch.ones(128))), ((h, h, pos), dict(q_out=h.float())), ((h, h, pos), dict(k_out=h[:, :2])),
                     ((h, h, pos), dict(q_out=h[:1].expand(3, 4, 128)))]:
        with pytest.raises(ValueError):
            dc.qk_norm_rope(*args, **kw)


@pytest.mark.parametrize("scale", [1e-60, 1e-46, 2.0 ** -127])
def test_a_scale_that_fp32_does_not_hold_is_refused(scale):
    """Rounded to 0 it would be taken for the default, 1 / sqrt(head_dim)."""
    q = torch.zeros((2, 3, 4, 128), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="scale"):
        dc.tree_attention(q, dc.KvCache(*_kv()), [0, 0], [3, 3], scale=scale)


@pytest.mark.parametrize("p", [[2 ** 32 - 1, 0], [-1, 2 ** 32], [-1, -2 ** 32], [-1, 2 ** 70]])
def test_parents_outside_32_bits_are_no_rows(p):
    """Cut to 32 bits they would be -1 and 0."""
    with pytest.raises((ValueError, dc.DepCapError)):
        dc.tree_mask([p])


def test_an_output_in_the_place_of_the_queries_has_their_strides():
    """As of qk_norm_rope: at other strides a row's output lies where another row's queries still are."""
    q = torch.zeros((2, 3, 4, 128), dtype=torch.bfloat16)
    c = dc.KvCache(*_kv())
    with pytest.raises(RuntimeError, match="no CPU path"):
        dc.tree_attention(q, c, [0, 0], [3, 3], out=q)
    with pytest.raises(ValueError, match="strides"):
        dc.tree_attention(q, c, [0, 0], [3, 3], out=q.view(2, 4, 3, 128).transpose(1, 2))

"""The operators around a cache on the GPU against 64 bits."""
import math
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import ops_ref as ref
import paper_2604_15750_b200 as dc

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, BF16, E4M3 = torch.float32, torch.bfloat16, torch.float8_e4m3fn


def gen(seed):
    return torch.Generator().manual_seed(seed)


def near(got, want, tol):
    got = got.detach().cpu().double()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    over = ((got - want).abs() - tol).nan_to_num(0)
    assert (over <= 0).all(), (float(over.max()), float(((got - want).abs() / tol.clamp(min=1e-300)).nan_to_num(0).max()))


def raw(t):
    return t.view(torch.uint8) if t.dtype == E4M3 else t


# ---- norm and rotation ------------------------------------------------------------------------------
ROPE = [  # dtype, rows, hq, hkv, hd, first position
    (BF16, 1, 32, 32, 128, 619), (BF16, 3, 28, 4, 128, 0), (BF16, 517, 32, 8, 128, 131000), (BF16, 65, 5, 1, 64, 2 ** 30),
    (F32, 48, 4, 4, 64, 64), (F32, 7, 3, 2, 128, 100001), (F32, 2, 1, 1, 2, 5), (BF16, 9, 3, 3, 6, 17), (F32, 5, 2, 1, 256, 4096),
    (BF16, 33, 7, 7, 256, 9), (BF16, 4, 0, 3, 96, 77), (F32, 4, 6, 0, 80, 77), (BF16, 6, 2, 2, 32, 3), (BF16, 300, 130, 11, 128, 8000),
]


def _rope_inputs(dtype, rows, hq, hkv, hd, first, seed=0):
    g = gen(seed)
    qkv = (torch.randn((rows, hq + 2 * hkv, hd), generator=g) * 3).to(dtype)
    gains = [(torch.rand(hd, generator=g) + 0.5).to(dtype) for _ in range(2)]
    pos = torch.arange(first, first + rows, dtype=torch.int32)
    return qkv, gains, pos


@pytest.mark.parametrize("dtype,rows,hq,hkv,hd,first", ROPE)
@pytest.mark.parametrize("with_gain", [True, False])
def test_qk_norm_rope(dtype, rows, hq, hkv, hd, first, with_gain):
    qkv, gains, pos = _rope_inputs(dtype, rows, hq, hkv, hd, first)
    x = qkv.to(DEV)
    gq, gk = gains if with_gain else (None, None)
    q, k = x[:, :hq], x[:, hq:hq + hkv]
    on = lambda t: None if t is None else t.to(DEV)
    oq, ok = dc.qk_norm_rope(q, k, pos.to(DEV), on(gq), on(gk), eps=1e-6, rope_theta=1e6)
    for got, part, gain in ((oq, qkv[:, :hq], gq), (ok, qkv[:, hq:hq + hkv], gk)):
        want, size = ref.rope(part, pos, gain, 1e-6, 1e6)
        near(got, want, ref.rope_tolerance(want, size, dtype))
    assert torch.equal(x.cpu(), qkv)


@pytest.mark.parametrize("dtype,hd,off,pad", [(BF16, 128, 0, 0), (BF16, 128, 1, 0), (BF16, 128, 0, 3), (F32, 64, 1, 5), (BF16, 64, 8, 8)])
def test_qk_norm_rope_in_place_and_odd_strides(dtype, hd, off, pad):
    """In place, rows that do not start on 16-byte boundaries, gaps between heads; what lies between is left as it was."""
    rows, hq, hkv = 37, 6, 2
    g = gen(1)
    buf = torch.randn((rows * (hq + hkv) * (hd + pad) + off,), generator=g).to(dtype)
    view = lambda t: t[off:].view(rows, hq + hkv, hd + pad)[..., :hd]
    x = buf.to(DEV)
    pos = torch.randint(0, 5000, (rows,), generator=g, dtype=torch.int32)
    gain = (torch.rand(hd, generator=g) + 0.5).to(dtype)
    q, k = view(x)[:, :hq], view(x)[:, hq:]
    oq, ok = dc.qk_norm_rope(q, k, pos.to(DEV), gain.to(DEV), gain.to(DEV), q_out=q, k_out=k)
    assert oq.data_ptr() == q.data_ptr()
    want, size = ref.rope(view(buf), pos, gain, 1e-5, 10000.0)
    near(view(x), want, ref.rope_tolerance(want, size, dtype))
    if pad:
        assert torch.equal(x.cpu()[off:].view(rows, hq + hkv, -1)[..., hd:], buf[off:].view(rows, hq + hkv, -1)[..., hd:])


def test_qk_norm_rope_keeps_nan_to_its_head():
    x = torch.randn((2, 4, 128), generator=gen(3)).to(BF16)
    x[1, 2, 5] = math.nan
    y, _ = dc.qk_norm_rope(x.to(DEV), x[:, :1].to(DEV), torch.zeros(2, dtype=torch.int32, device=DEV))
    bad = torch.isnan(y.cpu()).any(-1)
    assert bad[1, 2] and bad.sum() == 1


def test_qk_norm_rope_of_nothing():
    e = torch.empty((0, 4, 128), dtype=BF16, device=DEV)
    q, k = dc.qk_norm_rope(e, e, torch.empty(0, dtype=torch.int32, device=DEV))
    assert q.shape == e.shape


# ---- a cache written and read -------------------------------------------------------------------------
def _cache(layers, slots, heads, room, hd, dtype, seed=9):
    """a cache with something else in it already"""
    c = dc.KvCache.empty(layers, slots, heads, room, hd, dtype, DEV)
    g = gen(seed)
    for t in (c.k, c.v):
        if dtype == E4M3:
            raw(t).copy_(torch.randint(0, 120, t.shape, generator=g, dtype=torch.uint8))
        else:
            t.copy_(torch.randn(t.shape, generator=g))
    if dtype == E4M3:
        c.k_scale.copy_(torch.rand(c.k_scale.shape, generator=g) + 0.5)
        c.v_scale.copy_(torch.rand(c.v_scale.shape, generator=g) + 0.5)
    return c


def _given(rows, layout):
    """rows [layers, batch, n, heads, hd] on the device in a memory order of its own"""
    if layout == "rows":
        return rows.to(DEV)
    if layout == "cache":        # heads outside the keys, as in K caches
        return rows.transpose(2, 3).contiguous().to(DEV).transpose(2, 3)
    if layout == "across":       # keys contiguous, as in V caches; rows of 64 keys
        L, B, n, H, D = rows.shape
        t = torch.zeros((L, B, H, D, n + (-n) % 64), dtype=rows.dtype)
        t[..., :n] = rows.permute(0, 1, 3, 4, 2)
        return t.to(DEV).permute(0, 1, 4, 2, 3)[:, :, :n]
    if layout == "odd":          # neither on 16-byte boundaries
        L, B, n, H, D = rows.shape
        t = torch.zeros(L * B * n * H * (D + 1) + 1, dtype=rows.dtype)
        t[1:].view(L, B, n, H, D + 1)[..., :D] = rows
        return t.to(DEV)[1:].view(L, B, n, H, D + 1)[..., :D]
    if layout == "loose":        # no axis contiguous
        return torch.stack((rows, rows), -1).to(DEV)[..., 0]
    raise AssertionError(layout)


MOVES = [  # rows' type, held, layers, batch, rows, heads, hd, first positions, lengths
    (BF16, E4M3, 1, 1, 1, 2, 128, [0], [1]), (BF16, E4M3, 1, 1, 32, 4, 128, [512], [32]),
    (BF16, E4M3, 2, 3, 200, 3, 128, [0, 61, 130], [200, 0, 77]), (BF16, E4M3, 1, 2, 130, 1, 64, [63, 1], [130, 129]),
    (F32, E4M3, 1, 2, 70, 2, 64, [5, 64], [70, 64]), (F32, E4M3, 1, 1, 9, 1, 8, [3], [9]), (BF16, E4M3, 1, 1, 33, 2, 256, [31], [33]),
    (BF16, E4M3, 1, 2, 40, 2, 96, [8, 24], [40, 17]), (BF16, BF16, 2, 2, 150, 3, 128, [7, 0], [150, 3]), (F32, F32, 1, 1, 65, 2, 64, [64], [65]),
    (F32, F32, 1, 2, 20, 1, 24, [1, 2], [20, 19]), (BF16, E4M3, 3, 2, 256, 2, 128, [128, 0], [256, 255]), (F32, E4M3, 1, 1, 129, 2, 128, [120], [129]),
    (BF16, BF16, 1, 1, 128, 2, 128, [128], [128]),
]


@pytest.mark.parametrize("kl,vl", [("rows", "rows"), ("cache", "across"), ("odd", "odd"), ("loose", "across"), ("across", "loose")])
@pytest.mark.parametrize("dtype,held,L,B,n,H,D,pos,lens", MOVES)
def test_cache_write_and_read(dtype, held, L, B, n, H, D, pos, lens, kl, vl):
    room = (max(p + m for p, m in zip(pos, lens)) + 63) // 64 * 64 + 64
    c = _cache(L + 1, B + 1, H, room, D, held)
    before = [t.clone() if t is not None else None for t in (c.k, c.v, c.k_scale, c.v_scale)]
    g = gen(5)
    k, v = (((torch.randn((L, B, n, H, D), generator=g) * torch.exp2(torch.randint(-9, 9, (L, B, n, H, 1), generator=g))).to(dtype))
            for _ in range(2))
    k[0, 0, 0, 0] = 0     # a row of zeros
    dc.cache_write(c, _given(k, kl), _given(v, vl), pos, lens, layer=1)
    want = [t.cpu().clone() if t is not None else None for t in before]
    for b in range(B):
        p, m = pos[b], lens[b]
        for x, at, sc in ((k, 0, 2), (v, 1, 3)):
            rows = x[:, b, :m].transpose(1, 2)          # [layer, head, row, dim]
            if held == E4M3:
                rows, s = ref.quantised(rows)
                want[sc][1:, b, :, p:p + m] = s
                # and by the definition: off by half a step of the held value at most
                err = (rows.double() * s.double()[..., None] - x[:, b, :m].transpose(1, 2).double()).abs()
                xx = x[:, b, :m].transpose(1, 2).double().abs()
                assert (err <= torch.maximum(xx * 2.0 ** -4, s.double()[..., None] * 2.0 ** -10) + xx * 2.0 ** -22).all()
            if at == 0:
                raw(want[0])[1:, b, :, p:p + m] = raw(rows)
            else:
                raw(want[1])[1:, b, :, :, p:p + m] = raw(rows.contiguous()).transpose(2, 3)
    for got, w in zip((c.k, c.v, c.k_scale, c.v_scale), want):
        if w is not None:
            assert torch.equal(raw(got).cpu(), raw(w))
    # and back: what is held stands for held * scale, rounded once
    ko, vo = (_given(torch.full((L, B, n, H, D), 7.0, dtype=dtype), lay) for lay in (kl, vl))
    dc.cache_read(c, ko, vo, pos, lens, layer=1)
    for b in range(B):
        p, m = pos[b], lens[b]
        for got, at, sc in ((ko, want[0][1:, b, :, p:p + m], 2), (vo, want[1][1:, b, :, :, p:p + m].transpose(2, 3), 3)):
            x = at.float()
            if held == E4M3:
                x = x * want[sc][1:, b, :, p:p + m][..., None]
            assert torch.equal(got[:, b, :m].cpu(), x.transpose(1, 2).to(dtype))
            assert (got[:, b, m:] == 7).all()


@pytest.mark.parametrize("layout", ["rows", "across"])
def test_cache_write_of_values_that_are_not_finite(layout):
    """A row's scale goes by its finite values; infinities are held as +-448, NaN as NaN; the neighbours do not notice."""
    D, n = 128, 40
    x = torch.randn((1, 1, n, 2, D), generator=gen(2)).to(BF16)
    x[0, 0, 3, 0, 7], x[0, 0, 3, 0, 9], x[0, 0, 5, 1, 0] = math.inf, -math.inf, math.nan
    x[0, 0, 6, 1] = math.nan
    x[0, 0, 8, 0], x[0, 0, 9, 0] = 1e-38, 3e38
    c = _cache(1, 1, 2, 64, D, E4M3)
    dc.cache_write(c, _given(x, "rows"), _given(x, layout), [2])
    want, s = ref.quantised(x[0, 0].transpose(0, 1))
    for held, scale in ((c.k[0, 0, :, 2:2 + n], c.k_scale), (c.v[0, 0, :, :, 2:2 + n].transpose(1, 2), c.v_scale)):
        h, w = held.float().cpu(), want.float()
        assert torch.equal(torch.isnan(h), torch.isnan(w)) and torch.equal(h.nan_to_num(0), w.nan_to_num(0))
        assert torch.equal(scale[0, 0, :, 2:2 + n].cpu(), s)
    ko, vo = torch.zeros_like(x, device=DEV), torch.zeros_like(x, device=DEV)
    dc.cache_read(c, ko, vo, [2])
    assert torch.isnan(ko[0, 0, 6, 1]).all() and torch.isfinite(vo[0, 0, 4]).all()


def test_a_bf16_context_becomes_an_8_bit_one_and_comes_back():
    """KvCache.rows(): the arrays of DepCap.step into an 8-bit cache and back, other keys untouched."""
    plain, c = _cache(3, 2, 4, 192, 128, BF16), _cache(3, 2, 4, 256, 128, E4M3)
    before = [plain.k.clone(), plain.v.clone()]
    dc.cache_write(c, *plain.rows(), [0, 0], [150, 33])
    dc.cache_read(c, *plain.rows(), [0, 0], [150, 33])
    for got, old, tokens in ((plain.k, before[0], 3), (plain.v.transpose(3, 4), before[1].transpose(3, 4), 3)):
        for b, n in ((0, 150), (1, 33)):
            x = old[:, b, :, :n].float().cpu()
            held, s = ref.quantised(x)
            assert torch.equal(got[:, b, :, :n].cpu(), (held.float() * s[..., None]).to(BF16))
            assert torch.equal(got[:, b, :, n:], old[:, b, :, n:])


def test_keys_behind_two_to_the_31_values():
    """Offsets in a long cache pass 32 bits: the last keys of the last head of a cache of 2^32 + values a side."""
    c = dc.KvCache(torch.empty((1, 1, 260, 131072, 128), dtype=E4M3, device=DEV), torch.empty((1, 1, 260, 128, 131072), dtype=E4M3, device=DEV),
                   torch.ones((1, 1, 260, 131072), device=DEV), torch.ones((1, 1, 260, 131072), device=DEV))
    g = gen(4)
    x = torch.randn((1, 16, 260, 128), generator=g).to(BF16).to(DEV)
    y = torch.randn((1, 16, 260, 128), generator=g).to(BF16).to(DEV)
    at = 131072 - 16
    raw(c.k)[0, 0, 258:, :at] = 0
    raw(c.v)[0, 0, 258:, :, :at] = 0
    dc.cache_write(c, x, y, [at])
    ko, vo = torch.zeros_like(x), torch.zeros_like(y)
    dc.cache_read(c, ko, vo, [at])
    for got, given in ((ko, x), (vo, y)):
        held, s = ref.quantised(given.cpu())
        assert torch.equal(got.cpu(), (held.float() * s[..., None]).to(BF16))
    assert not raw(c.k)[0, 0, 259, :at].any() and not raw(c.v)[0, 0, 259, :, :at].any()
    q = torch.randn((1, 16, 260, 128), generator=g).to(BF16)
    out = dc.tree_attention(q.to(DEV), c, [at], [16])
    k = torch.cat((torch.zeros(1, at, 128), ko[0, :, 259:].cpu().transpose(0, 1).float()), 1)
    v = torch.cat((torch.zeros(1, at, 128), vo[0, :, 259:].cpu().transpose(0, 1).float()), 1)
    want, p = ref.tree(q[0, :, 259:], k, v, at, 16, None, 128 ** -0.5)
    tol = ref.tree_tolerance(q[0, :, 259:], k, v, p, want, 128 ** -0.5, BF16, c.v_scale[0, 0, 259:].cpu(), c.v[0, 0, 259:].cpu().transpose(1, 2).float(), True)
    near(out[0, :, 259:], want, tol)


# ---- attention of drafted rows --------------------------------------------------------------------------
TREES = [  # type of q, held, ctx_len, n_rows, max_rows, hq, hkv, hd, tree
    (BF16, E4M3, [512], [1], 1, 4, 4, 128, False), (BF16, E4M3, [0], [1], 1, 2, 2, 128, True), (BF16, BF16, [1], [1], 4, 2, 1, 128, True),
    (BF16, E4M3, [700, 0, 127, 128], [24, 24, 1, 0], 24, 4, 2, 128, True), (BF16, BF16, [700, 0, 127, 128], [24, 24, 1, 0], 24, 4, 2, 128, True),
    (BF16, E4M3, [1000], [64], 64, 7, 1, 128, True), (BF16, BF16, [1000], [64], 64, 7, 1, 128, False),
    (BF16, E4M3, [333, 60], [256, 190], 256, 4, 2, 128, True), (BF16, BF16, [333, 60], [256, 190], 256, 4, 2, 128, True),
    (BF16, E4M3, [5000], [3], 5, 2, 1, 128, True), (BF16, BF16, [5000], [3], 5, 2, 1, 128, True), (BF16, E4M3, [90, 200], [33, 65], 70, 3, 3, 128, True),
    (BF16, BF16, [127, 129], [17, 40], 40, 8, 8, 128, True), (BF16, E4M3, [2049], [9], 9, 56, 8, 128, True),
    (F32, F32, [64], [16], 16, 4, 4, 64, True), (F32, F32, [1000, 3], [5, 37], 40, 6, 2, 128, True), (F32, E4M3, [300], [20], 20, 4, 1, 64, True),
    (BF16, E4M3, [257], [12], 12, 4, 2, 64, True), (BF16, BF16, [257, 0], [12, 5], 12, 4, 2, 96, True), (F32, F32, [40], [10], 11, 2, 1, 256, False),
    (F32, F32, [500, 77], [33, 4], 33, 6, 2, 128, True), (F32, E4M3, [190], [70], 70, 3, 1, 128, True), (BF16, BF16, [200], [9], 9, 4, 4, 64, False),
    (F32, F32, [9], [3], 3, 2, 2, 8, True), (BF16, E4M3, [1500], [40], 40, 2, 1, 256, True),
]


def _tree_case(dtype, held, ctx, rows, most, hq, hkv, hd, tree, seed=11, spread=1.0):
    g = gen(seed)
    B = len(ctx)
    room = (max(c + r for c, r in zip(ctx, rows)) + 63) // 64 * 64
    c = _cache(2, B, hkv, room, hd, held)
    # the cache beyond the keys in use is NaN everywhere
    if held == E4M3:
        raw(c.k)[1].fill_(0x7F)
        raw(c.v)[1].fill_(0xFF)
        c.k_scale[1].fill_(math.nan)
        c.v_scale[1].fill_(math.inf)
    else:
        c.k[1].fill_(math.nan)
        c.v[1].fill_(math.inf)
    n = max(c + r for c, r in zip(ctx, rows))
    k, v = (torch.randn((B, n, hkv, hd), generator=g) * (torch.rand((B, n, hkv, 1), generator=g) + 0.5) for _ in range(2))
    if held != E4M3 or dtype == BF16:
        k, v = k.to(dtype), v.to(dtype)
    dc.cache_write(c, k.to(DEV), v.to(DEV), [0] * B, [x + r for x, r in zip(ctx, rows)], layer=1)
    q = (torch.randn((B, most, hq, hd), generator=g) * spread).to(dtype)
    mask = bools = None
    if tree:
        rng = np.random.RandomState(seed)
        parents = [[int(rng.randint(max(-1, i - 6), i)) if i else -1 for i in range(r)] for r in rows]
        mask = dc.tree_mask(parents, most)
        bools = torch.zeros((B, most, most), dtype=torch.bool)
        for b, ps in enumerate(parents):
            for i, p in enumerate(ps):
                if p >= 0:
                    bools[b, i] = bools[b, p]
                bools[b, i, i] = True
    return c, q, mask, bools


def _check_tree(c, layer, q, ctx, rows, bools, out, scale=None):
    hd, held = c.head_dim, c.dtype
    scale = hd ** -0.5 if scale is None else scale
    tc = q.dtype == BF16 and hd == 128
    for b, (x, r) in enumerate(zip(ctx, rows)):
        if r == 0:
            continue
        k, v = c.k[layer, b].float().cpu(), c.v[layer, b].float().cpu().transpose(1, 2)
        vs = v8 = None
        if held == E4M3:
            vs, v8 = c.v_scale[layer, b].cpu(), v
            k, v = k * c.k_scale[layer, b].cpu()[..., None], v * vs[..., None]
        qq = q[b].cpu()
        want, p = ref.tree(qq, k, v, x, r, None if bools is None else bools[b], scale)
        near(out[b, :r], want, ref.tree_tolerance(qq, k, v, p, want, scale, q.dtype, vs, v8, tc))


@pytest.mark.parametrize("dtype,held,ctx,rows,most,hq,hkv,hd,tree", TREES)
def test_tree_attention(dtype, held, ctx, rows, most, hq, hkv, hd, tree):
    c, q, mask, bools = _tree_case(dtype, held, ctx, rows, most, hq, hkv, hd, tree)
    out = torch.full(q.shape, 5.0, dtype=dtype, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    dc.tree_attention(q.to(DEV), c, ctx, rows, None if mask is None else mask.to(DEV), layer=1, out=out, status=status)
    _check_tree(c, 1, q, ctx, rows, bools, out)
    for b, r in enumerate(rows):
        assert (out[b, r:] == 5).all()
    assert int(status) == 0


@pytest.mark.parametrize("held", [E4M3, BF16])
@pytest.mark.parametrize("spread,scale", [(30.0, None), (1.0, 4.0), (1e-6, None), (1.0, 1e-4)])
def test_tree_attention_peaked_and_flat(held, spread, scale):
    ctx, rows = [1300, 40], [30, 30]
    c, q, mask, bools = _tree_case(BF16, held, ctx, rows, 30, 4, 2, 128, True, spread=spread)
    out = dc.tree_attention(q.to(DEV), c, ctx, rows, mask.to(DEV), layer=1, scale=scale)
    _check_tree(c, 1, q, ctx, rows, bools, out, scale)


@pytest.mark.parametrize("held", [E4M3, BF16])
def test_tree_attention_scores_that_climb(held):
    """Every tile of keys has larger scores than the one before: the running maximum moves all the time."""
    ctx, rows = [2000], [20]
    c, q, mask, bools = _tree_case(BF16, held, ctx, rows, 20, 2, 1, 128, True)
    n = 2020
    k = torch.ones((1, n, 1, 128)) * (torch.arange(n).float() / n * 12)[None, :, None, None] + torch.randn((1, n, 1, 128), generator=gen(1)) * 0.1
    v = torch.randn((1, n, 1, 128), generator=gen(2)) * torch.exp2(torch.randint(-6, 6, (1, n, 1, 1), generator=gen(3)))
    dc.cache_write(c, k.to(BF16).to(DEV), v.to(BF16).to(DEV), [0], layer=1)
    q = (q.float().abs() + 0.5).to(BF16)
    out = dc.tree_attention(q.to(DEV), c, ctx, rows, mask.to(DEV), layer=1)
    _check_tree(c, 1, q, ctx, rows, bools, out)


def _drawn(seed, longest, most):
    rng = np.random.RandomState(seed)
    B = int(rng.randint(1, 5))
    rows = [int(rng.randint(1, most + 1)) for _ in range(B)]
    ctx = [int(2 ** rng.uniform(0, math.log2(longest))) if rng.rand() < 0.85 else 0 for _ in range(B)]
    hkv = int(rng.choice([1, 2, 4]))
    return ctx, rows, max(rows) + int(rng.randint(0, 3)), hkv * int(rng.choice([1, 2, 4, 7])), hkv, bool(rng.rand() < 0.7)


@pytest.mark.parametrize("seed", range(16))
@pytest.mark.parametrize("dtype,held,hd", [(BF16, E4M3, 128), (BF16, BF16, 128), (F32, F32, 64), (F32, F32, 128), (BF16, BF16, 64), (F32, E4M3, 64)])
def test_tree_attention_drawn_shapes(dtype, held, hd, seed):
    """Whatever width, stretch and join the sizes lead to: one row to 256, one key to thousands, lengths far apart."""
    big = hd == 128 and dtype == BF16
    ctx, rows, most, hq, hkv, tree = _drawn(100 + seed, (8000 if seed % 4 == 0 else 1500) if big else 1200, (256, 40, 6, 1)[seed % 4])
    c, q, mask, bools = _tree_case(dtype, held, ctx, rows, most, hq, hkv, hd, tree, seed=seed)
    out = dc.tree_attention(q.to(DEV), c, ctx, rows, None if mask is None else mask.to(DEV), layer=1)
    _check_tree(c, 1, q, ctx, rows, bools, out)


@pytest.mark.parametrize("held,hd", [(E4M3, 128), (BF16, 128), (BF16, 64)])
def test_tree_attention_rows_without_a_key_and_any_mask(held, hd):
    """Masks that are no tree: bits above the diagonal, rows that see nothing (zeros), bits beyond the rows (not looked at)."""
    ctx, rows, most = [0, 130], [50, 50], 50
    c, q, _, _ = _tree_case(BF16, held, ctx, rows, most, 4, 2, hd, False)
    bools = torch.rand((2, most, most), generator=gen(8)) < 0.3
    bools[0, 7] = bools[0, 49] = False
    bools[1, 3] = False
    words = torch.zeros((2, most, 2), dtype=torch.int64)
    for j in range(most):
        words[..., j // 32] |= bools[..., j].long() << (j % 32)
    words[..., 1] |= 0xFFFC0000          # beyond row 49
    mask = torch.where(words >= 2 ** 31, words - 2 ** 32, words).to(torch.int32)
    out = dc.tree_attention(q.to(DEV), c, ctx, rows, mask.to(DEV), layer=1)
    _check_tree(c, 1, q, ctx, rows, bools, out)
    assert (out[0, 7] == 0).all() and (out[0, 49] == 0).all()


@pytest.mark.parametrize("held,hd", [(E4M3, 128), (BF16, 128), (BF16, 64)])
@pytest.mark.parametrize("where", ["k", "v"])
def test_tree_attention_values_that_are_not_finite_stay_with_the_rows_that_see_them(held, hd, where):
    ctx, rows = [100], [40]
    c, q, mask, bools = _tree_case(BF16, held, ctx, rows, 40, 4, 2, hd, True)
    j, clean = 5, None
    bad = torch.randn((1, 1, 2, hd), generator=gen(1)).to(BF16)
    bad[0, 0, :, 3] = math.nan
    good = torch.randn((1, 1, 2, hd), generator=gen(2)).to(BF16)
    ref_out = dc.tree_attention(q.to(DEV), c, ctx, rows, mask.to(DEV), layer=1)
    dc.cache_write(c, (bad if where == "k" else good).to(DEV), (bad if where == "v" else good).to(DEV), [ctx[0] + j], layer=1)
    out = dc.tree_attention(q.to(DEV), c, ctx, rows, mask.to(DEV), layer=1).cpu()
    for r in range(40):
        if bools[0, r, j]:
            assert torch.isnan(out[0, r, :, 3]).all()
        else:
            assert torch.equal(out[0, r], ref_out[0, r].cpu())
    assert bools[0, :, j].any() and not bools[0, :, j].all()


@pytest.mark.parametrize("held,hd", [(E4M3, 128), (BF16, 128), (BF16, 64), (BF16, 96), (E4M3, 8)])
def test_tree_attention_a_value_that_is_not_finite_behind_a_probability_of_zero(held, hd):
    """A drafted key far below the others' scores: rows that see it are NaN where its V is, the others as they were."""
    c, q, mask, bools = _tree_case(BF16, held, [100], [40], 40, 4, 2, hd, True)
    q = torch.full_like(q, 4.0)
    key, value = torch.full((1, 1, 2, hd), -64.0, dtype=BF16), torch.ones((1, 1, 2, hd), dtype=BF16)
    dc.cache_write(c, key.to(DEV), value.to(DEV), [105], layer=1)
    before = dc.tree_attention(q.to(DEV), c, [100], [40], mask.to(DEV), layer=1).cpu()
    value[..., 3] = math.nan
    dc.cache_write(c, key.to(DEV), value.to(DEV), [105], layer=1)
    out = dc.tree_attention(q.to(DEV), c, [100], [40], mask.to(DEV), layer=1).cpu()
    assert not torch.isnan(before).any() and bools[0, :, 5].any()
    for r in range(40):
        if bools[0, r, 5]:
            assert torch.isnan(out[0, r, :, 3]).all()
        else:
            assert torch.equal(out[0, r], before[0, r])


@pytest.mark.parametrize("held,hd", [(E4M3, 128), (BF16, 128), (F32, 64)])
def test_tree_attention_strides_and_bases(held, hd):
    """q and out as slices of larger tensors, out head by head; arrays off 16-byte boundaries."""
    dtype = F32 if held == F32 else BF16
    ctx, rows = [300, 41], [19, 7]
    c, q, mask, bools = _tree_case(dtype, held, ctx, rows, 19, 6, 3, hd, True)
    wide = torch.randn((2, 19, 12, hd + 8), generator=gen(1)).to(dtype).to(DEV)
    wide[:, :, 3:9, :hd] = q.to(DEV)
    heads = torch.full((2, 6, 19, hd), 3.0, dtype=dtype, device=DEV)
    dc.tree_attention(wide[:, :, 3:9, :hd], c, ctx, rows, mask.to(DEV), layer=1, out=heads.transpose(1, 2))
    _check_tree(c, 1, q, ctx, rows, bools, heads.transpose(1, 2))
    off = torch.zeros(q.numel() + 1, dtype=dtype, device=DEV)[1:].view(q.shape)
    off.copy_(q)
    out = torch.zeros(q.numel() + 1, dtype=dtype, device=DEV)[1:].view(q.shape)
    dc.tree_attention(off, c, ctx, rows, mask.to(DEV), layer=1, out=out)
    _check_tree(c, 1, q, ctx, rows, bools, out)
    shift = lambda t: torch.cat((raw(t).new_zeros(1), raw(t).flatten()))[1:].view(t.dtype).view(t.shape) if t is not None else None
    moved = dc.KvCache(shift(c.k), shift(c.v), c.k_scale, c.v_scale)
    out = dc.tree_attention(q.to(DEV), moved, ctx, rows, mask.to(DEV), layer=1)
    _check_tree(c, 1, q, ctx, rows, bools, out)


# ---- together, and how calls go with one another ----------------------------------------------------------
@pytest.mark.parametrize("held", [E4M3, BF16])
def test_a_layer_of_drafted_rows(held):
    """Projections -> norm and rotation -> into the cache -> attention, then the accepted rows behind the context and one
    more row: as a caller drives a layer, against 64 bits of the whole chain but the cache's own rounding."""
    B, R, hq, hkv, hd = 2, 12, 8, 2, 128
    ctx = [200, 77]
    c, _, _, _ = _tree_case(BF16, held, ctx, [0, 0], R + 4, hq, hkv, hd, False)
    big = dc.KvCache.empty(2, B, hkv, 320, hd, held, DEV)
    for name in ("k", "k_scale"):
        if getattr(c, name) is not None:
            raw(getattr(big, name))[:, :, :, :c.max_ctx] = raw(getattr(c, name))
    raw(big.v)[..., :c.max_ctx] = raw(c.v)
    if held == E4M3:
        big.v_scale[..., :c.max_ctx] = c.v_scale
    g = gen(6)
    qkv = torch.randn((B, R, hq + 2 * hkv, hd), generator=g).to(BF16).to(DEV)
    gain = (torch.rand(hd, generator=g) + 0.5).to(BF16).to(DEV)
    parents = [[-1, 0, 0, 1, 1, 2, 3, 3, 4, 5, 8, 8]] * B
    depth = [0, 1, 1, 2, 2, 2, 3, 3, 3, 3, 4, 4]
    pos = torch.tensor([[x + d for d in depth] for x in ctx], dtype=torch.int32, device=DEV)
    flat = qkv.view(B * R, -1, hd)
    q, k = dc.qk_norm_rope(flat[:, :hq], flat[:, hq:hq + hkv], pos.view(-1), gain, gain)
    q, k, v = q.view(B, R, hq, hd), k.view(B, R, hkv, hd), qkv[:, :, hq + hkv:]
    dc.cache_write(big, k, v, ctx, layer=1)
    mask = dc.tree_mask(parents).to(DEV)
    out = dc.tree_attention(q, big, ctx, [R] * B, mask, layer=1)
    bools = torch.zeros((B, R, R), dtype=torch.bool)
    for i, p in enumerate(parents[0]):
        if p >= 0:
            bools[:, i] = bools[:, p]
        bools[:, i, i] = True
    _check_tree(big, 1, q, ctx, [R] * B, bools, out)
    # rows 0, 1, 4, 8 are accepted: they go behind the context in that order, and are plain context for the next row
    path = [0, 1, 4, 8]
    dc.cache_write(big, k[:, path], v[:, path], ctx, layer=1)
    after = dc.tree_attention(q[:, 8:9], big, [x + 3 for x in ctx], [1] * B, layer=1)
    _check_tree(big, 1, q[:, 8:9], [x + 3 for x in ctx], [1] * B, None, after)
    tol = 2 * ref.HALF[BF16] * out[:, 8].abs().float() + 2.0 ** -7       # the same sums in another order, each within its tolerance
    assert ((after[:, 0].float() - out[:, 8].float()).abs() <= tol).all()


@pytest.mark.parametrize("held", [E4M3, BF16])
def test_calls_on_other_streams_in_graphs_and_twice(held):
    """The same bits from the default stream, another one, a graph (replayed with new inputs), and two calls at once."""
    ctx, rows = [900, 333], [24, 11]
    c, q, mask, bools = _tree_case(BF16, held, ctx, rows, 24, 8, 4, 128, True)
    qd, md = q.to(DEV), mask.to(DEV)
    first = dc.tree_attention(qd, c, ctx, rows, md, layer=1)
    assert torch.equal(first, dc.tree_attention(qd, c, ctx, rows, md, layer=1))
    torch.cuda.synchronize()
    side = [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.zeros_like(qd) for _ in side]
    torch.cuda.synchronize()
    outs = [dc.tree_attention(qd, c, ctx, rows, md, layer=1, stream=s, out=o) for s, o in zip(side, outs)]
    torch.cuda.synchronize()
    assert all(torch.equal(o, first) for o in outs)
    pos = torch.arange(48, dtype=torch.int32, device=DEV)
    graph, out, kv = torch.cuda.CUDAGraph(), torch.zeros_like(qd), torch.zeros((2, 24, 4, 128), dtype=BF16, device=DEV)
    qin = qd.clone()
    with torch.cuda.graph(graph):
        qn, _ = dc.qk_norm_rope(qin.view(48, 8, 128), kv.view(48, 4, 128), pos)
        dc.cache_write(c, kv, kv, ctx, rows, layer=1)
        dc.tree_attention(qn.view(2, 24, 8, 128), c, ctx, rows, md, layer=1, out=out)
    for seed in (1, 2):
        x = torch.randn(qd.shape, generator=gen(seed)).to(BF16)
        kv.copy_(torch.randn(kv.shape, generator=gen(seed + 9)))
        qin.copy_(x)
        out.zero_()
        graph.replay()
        got = out.clone()
        qn, _ = dc.qk_norm_rope(qin.view(48, 8, 128), kv.view(48, 4, 128), pos)
        dc.cache_write(c, kv, kv, ctx, rows, layer=1)
        assert torch.equal(got, dc.tree_attention(qn.view(2, 24, 8, 128), c, ctx, rows, md, layer=1))
        _check_tree(c, 1, qn.view(2, 24, 8, 128), ctx, rows, bools, got)


def test_outputs_made_for_a_call_on_another_stream_belong_to_that_stream():
    """The current stream is busy when the call is made: nothing of the output may wait for it."""
    c, q, mask, _ = _tree_case(BF16, E4M3, [200], [24], 24, 8, 4, 128, True)
    qd, md = q.to(DEV), mask.to(DEV)
    h, pos = qd[0], torch.arange(24, dtype=torch.int32, device=DEV)
    want, turned = dc.tree_attention(qd, c, [200], [24], md, layer=1), dc.qk_norm_rope(h, h, pos)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(3):
        torch.cuda._sleep(20_000_000)        # (10 ms)
        got, (a, b) = dc.tree_attention(qd, c, [200], [24], md, layer=1, stream=side), dc.qk_norm_rope(h, h, pos, stream=side)
        torch.cuda.synchronize()
        assert torch.equal(got, want) and torch.equal(a, turned[0]) and torch.equal(b, turned[1])


FIRST = """
import torch, paper_2604_15750_b200 as dc
c = dc.KvCache.empty(1, 2, 4, 4096, 128, dtype=torch.float8_e4m3fn)
x, q = (torch.randn(s, device="cuda").to(torch.bfloat16) for s in ((2, 300, 4, 128), (2, 24, 8, 128)))
pos, mask = torch.arange(48, dtype=torch.int32, device="cuda"), dc.tree_mask([[-1] + list(range(23))] * 2).cuda()
out, qo, ko = torch.zeros_like(q), torch.zeros_like(q), torch.zeros((48, 4, 128), dtype=torch.bfloat16, device="cuda")
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    dc.cache_write(c, x, x, [0, 0])
    dc.qk_norm_rope(q.view(48, 8, 128), ko, pos, q_out=qo.view(48, 8, 128), k_out=ko)
    dc.tree_attention(qo, c, [3000, 100], [24, 24], mask, out=out)
g.replay()
got = out.clone()
dc.tree_attention(qo, c, [3000, 100], [24, 24], mask, out=out)
assert torch.equal(got, out) and out.abs().sum() > 0
"""


def test_the_first_calls_of_a_process_may_be_captured():
    """What a kernel's first launch sets up (shared memory, places of clusters, modules) is no work on the stream."""
    r = subprocess.run([sys.executable, "-c", FIRST], cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))), capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stderr[-2000:]


def test_a_workspace_of_the_callers_own():
    ctx, rows = [6000], [4]
    c, q, mask, bools = _tree_case(BF16, E4M3, ctx, rows, 4, 2, 1, 128, True)
    need = dc.tree_attention_workspace(q.to(DEV), c, ctx, rows)
    assert need > 0
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device=DEV)
    out = dc.tree_attention(q.to(DEV), c, ctx, rows, mask.to(DEV), layer=1, workspace=ws)
    _check_tree(c, 1, q, ctx, rows, bools, out)
    with pytest.raises(dc.DepCapError):
        dc.tree_attention(q.to(DEV), c, ctx, rows, mask.to(DEV), layer=1, workspace=ws[:need - 16])


@pytest.mark.parametrize("held", [E4M3, BF16])
@pytest.mark.parametrize("ctx,rows,hq,hkv", [([5000, 2900], [200, 256], 8, 4), ([4100], [3], 64, 1), ([700, 699], [2, 1], 66, 2)])
def test_tree_attention_many_lines_of_a_kv_head(held, ctx, rows, hq, hkv):
    """Over 64 rows x heads of a kv head with work for every SM (128 a CTA), a large group, a group of odd size."""
    most = max(rows)
    c, q, mask, bools = _tree_case(BF16, held, ctx, rows, most, hq, hkv, 128, True)
    out = dc.tree_attention(q.to(DEV), c, ctx, rows, mask.to(DEV), layer=1)
    _check_tree(c, 1, q, ctx, rows, bools, out)


@pytest.mark.parametrize("held,hd", [(E4M3, 128), (BF16, 128), (E4M3, 64)])
@pytest.mark.parametrize("ctx", [1000, 40000])
def test_values_that_are_not_finite_in_a_context_cut_into_stretches(held, hd, ctx):
    """As above, where a cluster (1000 keys) or a second launch (40000) joins the stretches; and K of the same key."""
    rows = [40]
    c, q, mask, bools = _tree_case(BF16, held, [ctx], rows, 40, 2, 1, hd, True)
    ref_out = dc.tree_attention(q.to(DEV), c, [ctx], rows, mask.to(DEV), layer=1)
    _check_tree(c, 1, q, [ctx], rows, bools, ref_out)
    for bad_k in (False, True):
        j = 5
        x = torch.randn((2, 1, 1, 1, hd), generator=gen(1)).to(BF16)
        x[0 if bad_k else 1, ..., 3] = math.inf if held == BF16 and not bad_k else math.nan
        dc.cache_write(c, x[0].to(DEV), x[1].to(DEV), [ctx + j], layer=1)
        out = dc.tree_attention(q.to(DEV), c, [ctx], rows, mask.to(DEV), layer=1).cpu()
        for r in range(40):
            if bools[0, r, j]:
                assert not torch.isfinite(out[0, r, :, 3]).any()
            else:
                assert torch.equal(out[0, r], ref_out[0, r].cpu())


def test_keys_with_a_scale_of_zero_count():
    """A row of zeros that came with a scale of 0 is a key like any other: its probability is in the sum."""
    ctx, rows = [200], [8]
    c, q, mask, bools = _tree_case(BF16, E4M3, ctx, rows, 8, 4, 2, 128, True)
    for t in (c.k, c.k_scale, c.v_scale):
        raw(t)[1, 0, :, 50:90] = 0
    raw(c.v)[1, 0, :, :, 50:90] = 0
    out = dc.tree_attention(q.to(DEV), c, ctx, rows, mask.to(DEV), layer=1)
    _check_tree(c, 1, q, ctx, rows, bools, out)


def test_two_writes_at_once_side_by_side():
    """Neighbouring keys of one slot written on two streams: no write touches a byte of the other's."""
    n, cut = 150, 77
    c = _cache(2, 1, 4, 192, 128, E4M3)
    x = torch.randn((2, 1, n, 4, 128), generator=gen(1)).to(BF16).to(DEV)
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(5):
        dc.cache_write(c, x[:, :, :cut], x[:, :, :cut], [3], stream=s1)
        dc.cache_write(c, x[:, :, cut:], x[:, :, cut:], [3 + cut], stream=s2)
    torch.cuda.synchronize()
    held, s = ref.quantised(x[:, 0].transpose(1, 2).cpu())
    assert torch.equal(raw(c.k[:, 0, :, 3:3 + n]).cpu(), raw(held))
    assert torch.equal(raw(c.v[:, 0, :, :, 3:3 + n]).cpu(), raw(held).transpose(2, 3))
    assert torch.equal(c.v_scale[:, 0, :, 3:3 + n].cpu(), s)


def test_a_prefilled_context_goes_through_8_bits_into_a_step():
    """prefill -> 8-bit cache -> the arrays of a step -> step: as with the context rounded on the host."""
    from paper_2604_15750_b200 import inputs
    wl = inputs.Workload("ops_bf16", 2, 256, 2, 2, 128, 512, 2048, "bf16", 2, 64, 128, 16, 32, 64, 4243)
    eng = dc.DepCap.from_workload(wl, inputs.make_weights(wl, DEV), max_last=128)
    tok = inputs.make_tokens(wl)
    kv = dc.KvCache.empty(2, 2, 2, 128, 128, BF16, DEV)
    ids = torch.zeros((2, 128), dtype=torch.int32, device=DEV)
    ids[:, :120] = tok["prompt"][:, :120].to(DEV)
    lens = [120, 77]
    assert not eng.prefill(kv.k, kv.v, ids, lens).any()
    c = dc.KvCache.empty(2, 2, 2, 192, 128, E4M3, DEV)
    dc.cache_write(c, *kv.rows(), [0, 0], lens)
    want_k, want_v = kv.k.clone().cpu(), kv.v.clone().cpu()
    back = dc.KvCache(kv.k.clone(), kv.v.clone())
    dc.cache_read(c, *back.rows(), [0, 0], lens)
    for b, n in enumerate(lens):
        h, s = ref.quantised(want_k[:, b, :, :n])
        want_k[:, b, :, :n] = (h.float() * s[..., None]).to(BF16)
        h, s = ref.quantised(want_v[:, b, :, :, :n].transpose(2, 3))
        want_v[:, b, :, :, :n] = (h.float() * s[..., None]).to(BF16).transpose(2, 3)
    assert torch.equal(back.k.cpu(), want_k) and torch.equal(back.v.cpu(), want_v)
    last = torch.zeros((2, 128), dtype=torch.int32, device=DEV)
    last[:, :16] = tok["last_ids"].to(DEV)
    win = tok["win_ids"].to(DEV)
    res = []
    for k, v in ((back.k, back.v), (want_k.to(DEV), want_v.to(DEV))):
        out = eng.step(k, v, lens, last, [16, 16], win, [32, 32], [64, 64])
        eng.synchronize()
        res.append({n: out[n].clone() for n in ("pred_id", "conf", "entropy", "influence", "block_len", "status")})
    assert not res[0]["status"].any()
    for n in res[0]:
        assert torch.equal(res[0][n], res[1][n]), n
    eng.close()


@pytest.mark.parametrize("far,spread", [(64.0, 0), (3000.0, 30), (1.0, 60)])
def test_tree_attention_outliers(far, spread):
    """One channel of the queries far above the others, rows of V whose sizes (and scales) lie 2^spread apart either way."""
    ctx, rows = [700], [21]
    c, q, mask, bools = _tree_case(BF16, E4M3, ctx, rows, 21, 4, 2, 128, True)
    n = 721
    k = torch.randn((1, n, 2, 128), generator=gen(1))
    k[..., 5] /= far
    v = torch.randn((1, n, 2, 128), generator=gen(2)) * torch.exp2(torch.randint(-spread, spread + 1, (1, n, 2, 1), generator=gen(3)).float())
    dc.cache_write(c, k.to(BF16).to(DEV), v.to(BF16).to(DEV), [0], layer=1)
    q = q.float()
    q[..., 5] *= far
    q = q.to(BF16)
    out = dc.tree_attention(q.to(DEV), c, ctx, rows, mask.to(DEV), layer=1)
    kk, v8 = c.k[1, 0].float().cpu() * c.k_scale[1, 0].cpu()[..., None], c.v[1, 0].float().cpu().transpose(1, 2)
    vs = c.v_scale[1, 0].cpu()
    vv = v8.double() * vs.double()[..., None]
    want, p = ref.tree(q[0], kk, vv, 700, 21, bools[0], 128 ** -0.5)
    near(out[0], want, ref.tree_tolerance(q[0], kk, vv, p, want, 128 ** -0.5, BF16, vs, v8, True, outliers=True))

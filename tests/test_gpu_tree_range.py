"""Attention of drafted rows over an 8-bit cache on the tensor cores: what is far below a row's largest value still counts."""
import math

import pytest
import torch

import ops_ref as ref
import paper_2604_15750_b200 as dc

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16, E4M3 = torch.bfloat16, torch.float8_e4m3fn


def _tolerance(q, k, v8, vs, p, o, scale):
    """tree_tolerance's terms of the scores, the sums, the probabilities' 8 bits (2^-8 at most) and the output's rounding.  Beside them
    a probability x scale of V is not held more finely than 2^-27 of the row's largest: it is scaled until the largest is 2^10 at
    least, and its last part is rounded to multiples of 2^-16, half of which is 2^-17."""
    tol = ref.tree_tolerance(q, k, v8.double() * vs.double()[..., None], p, o, scale, BF16, tensor_cores=True)
    group = o.shape[1] // k.shape[0]
    for h in range(o.shape[1]):
        n = p.shape[-1]
        peak = (p[h] * vs[h // group, :n].double()).amax(-1, keepdim=True)
        tol[:, h] += 2.0 ** -27 * peak * v8[h // group, :n].double().abs().sum(0)
    return tol


@pytest.mark.parametrize("rows,B,H", [(8, 8, 37), (64, 4, 37), (128, 4, 37)])      # 32, 64, 128 lines; a unit for every place of the SMs
@pytest.mark.parametrize("keys", [4096, 16000])
@pytest.mark.parametrize("below", [15.0, 17.2, 20.0])
@pytest.mark.parametrize("first", [0, 700])
def test_a_flat_tail_far_below_one_key_counts(rows, B, H, keys, below, first):
    """One key 2^below times as probable as each of the others, whose V have a mean: together they are up to a third of the
    row, and what each of them loses has the same sign."""
    g = torch.Generator().manual_seed(int(below * 10) + keys)
    u, scale = torch.randn(128, generator=g) * 0.25, 128 ** -0.5
    u[0] = 0
    k = u.repeat(keys, 1)
    k[first, 0] = below / math.log2(math.e) / scale / 8        # (q's dim 0 is 8)
    v = 1 + 0.3 * torch.randn((keys, 128), generator=g)
    v[first] = -1 + 0.3 * torch.randn(128, generator=g)
    q = torch.randn((rows, 128), generator=g)
    q[:, 0] = 8
    k, v, q = k.to(BF16), v.to(BF16), q.to(BF16)
    c = dc.KvCache.empty(1, B, H, (keys + 63) // 64 * 64, 128, E4M3, DEV)
    spread = lambda t: t.to(DEV)[None, :, None].expand(B, -1, H, -1)
    ctx = keys - rows
    dc.cache_write(c, spread(k), spread(v), [0] * B)
    out = dc.tree_attention(spread(q).contiguous(), c, [ctx] * B, [rows] * B)
    held = lambda t: t[0, :1, :1].float().cpu()
    k8, v8, ks, vs = held(c.k)[0], held(c.v)[0].transpose(1, 2), held(c.k_scale)[0], held(c.v_scale)[0]
    k8, v8, ks, vs = k8[:, :keys], v8[:, :keys], ks[:, :keys], vs[:, :keys]
    kk = k8.double() * ks.double()[..., None]
    vv = v8.double() * vs.double()[..., None]
    p = torch.softmax(q.double() @ kk[0].T * scale, -1)
    o = (p @ vv[0])[:, None]
    assert 2.0 ** (below - 1) < float((p[:, first] / p[:, -1]).mean()) < 2.0 ** (below + 1)
    tol = _tolerance(q[:, None], kk, v8, vs, p[None], o, scale)
    assert torch.equal(out, out[:1, :, :1].expand_as(out))
    over = (out[0, :, :1].double().cpu() - o).abs() / tol
    assert (over <= 1).all(), float(over.max())


@pytest.mark.parametrize("rows", [8, 64, 128])
def test_small_dims_of_a_query_beside_a_large_one_are_exact(rows):
    """A query's dims down to 2^-13 of its largest one are held exactly, as sums of two 8-bit numbers: half of the keys have the dims
    with x = 2^-10 (1 + 2^-7) of the largest, half those with 2^-10 of it, and only what x has more decides between them."""
    keys, scale = 512, 128 ** -0.5
    q = torch.zeros((rows, 128))
    q[:, 0], q[:, 1:64], q[:, 64:127] = 2.0 ** 13, 8 * (1 + 2.0 ** -7), 8
    sign = torch.randint(0, 2, (rows, 1), generator=torch.Generator().manual_seed(1)) * 2 - 1
    q = (q * sign).to(BF16)
    k = torch.zeros((keys, 128))
    k[0::2, 1:64] = k[1::2, 64:127] = 1
    v = torch.ones((keys, 128))
    v[1::2] = -1
    c = dc.KvCache.empty(1, 1, 1, keys, 128, E4M3, DEV)
    shape = lambda t: t.to(BF16).to(DEV)[None, :, None]
    dc.cache_write(c, shape(k), shape(v), [0])
    out = dc.tree_attention(shape(q).contiguous(), c, [keys - rows], [rows])[0].double().cpu()
    kk = c.k[0, 0].double().cpu() * c.k_scale[0, 0].double().cpu()[..., None]
    v8, vs = c.v[0, 0].float().cpu().transpose(1, 2), c.v_scale[0, 0].cpu()
    p = torch.softmax(q.double() @ kk[0].T * scale, -1)
    o = (p @ (v8[0].double() * vs[0].double()[:, None]))[:, None]
    assert float(o.abs().min()) > 0.15
    over = (out - o).abs() / _tolerance(q[:, None], kk, v8, vs, p[None], o, scale)
    assert (over <= 1).all(), float(over.max())

"""The operators around a cache in 64 bits (numpy / torch on the CPU), and how far a kernel may be from them.

Roundings count half a step of their type relative to the value: fp32 2^-24, bf16 2^-8, e4m3 2^-4 (or half its least step,
2^-10, below the normal range)."""
import math

import torch

U32, HALF = 2.0 ** -24, {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def rope(x, pos, gain, eps, theta):
    """x [rows, heads, hd] -> (value, sum of the magnitudes that a value is the difference of), 64 bits"""
    x = x.double()
    hd = x.shape[-1]
    y = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    if gain is not None:
        y = y * gain.double()
    ang = pos.double()[:, None, None] * theta ** (-2.0 * torch.arange(hd // 2, dtype=torch.float64) / hd)
    c, s = ang.cos(), ang.sin()
    a, b = y.chunk(2, -1)
    return torch.cat((a * c - b * s, b * c + a * s), -1), torch.cat((a.abs() + b.abs(),) * 2, -1)


def rope_tolerance(ref, size, dtype):
    """Beside the output's rounding: mean of squares (at most hd/32 + 5 sums and a division), square root and reciprocal (3),
    two products, cos and sin (2 and what rounding an angle of up to pi to 24 bits moves them, pi), a product and a sum: under 30
    roundings of 2^-24 of each of the two terms."""
    return HALF[dtype] * ref.abs() + 30 * U32 * size


def quantised(x):
    """rows x [..., hd] -> (held values, scales) by the rule of an e4m3 cache, operation by operation in fp32"""
    x = x.float()
    a = torch.where(torch.isfinite(x), x.abs(), torch.zeros_like(x)).amax(-1)
    s = torch.maximum(a / 448, torch.tensor(2.0 ** -80))
    y = torch.nan_to_num(x * (1 / s)[..., None], nan=math.nan, posinf=448.0, neginf=-448.0).clamp(-448, 448)
    return y.to(torch.float8_e4m3fn), s


def tree(q, k, v, ctx, rows, mask, scale):
    """q [R, hq, hd], k and v [hkv, keys, hd] of one sequence in 64 bits, mask bool [R, rows] or None.
    -> o, probabilities [hq, R, keys]"""
    R, hq, hd = q.shape
    group = hq // k.shape[0]
    sees = torch.zeros((rows, ctx + rows), dtype=torch.bool)
    sees[:, :ctx] = True
    sees[:, ctx:] = True if mask is None else mask[:rows, :rows]
    o, p = torch.zeros((rows, hq, hd), dtype=torch.float64), torch.zeros((hq, rows, ctx + rows), dtype=torch.float64)
    any_ = sees.any(-1)
    for h in range(hq):
        z = (q[:rows, h].double() @ k[h // group, :ctx + rows].double().T) * scale
        z = z.masked_fill(~sees, -math.inf)
        w = torch.softmax(z[any_], -1) if bool(any_.any()) else z[any_]
        p[h, any_] = w
        # (what a row does not see has no part in it, whatever it is)
        vv = v[h // group, :ctx + rows].double()
        for r in torch.nonzero(any_).flatten().tolist():
            o[r, h] = p[h, r][sees[r]] @ vv[sees[r]]
    return o, p


def tree_tolerance(q, k, v, p, o, scale, dtype, vs=None, v8=None, tensor_cores=False, outliers=False):
    """[rows, hq, hd].  outliers: queries against an 8-bit cache are held to 2^-18 of a row's largest value, which counts where other
    values are 2^10 below it.  A score z = scale * q.k is off by at most (hd + 4) roundings of the sum of its terms' magnitudes (on the
    tensor cores, whose sums drop bits instead of rounding them, twice that), a probability by twice that relative (its own
    score and the sum's), the sum over n keys by n roundings.  On the tensor cores a probability is rounded to 8 bits (2^-8
    at most), and against an 8-bit cache not more finely than 2^-17 of the largest probability x scale of V."""
    rows, hq, hd = o.shape
    group = hq // k.shape[0]
    tol = torch.zeros_like(o)
    n = p.shape[-1]
    for h in range(hq):
        kk, vv = k[h // group, :n].double().nan_to_num(0, 0, 0).abs(), v[h // group, :n].double().nan_to_num(0, 0, 0).abs()
        size = (q[:rows, h].double().abs() @ kk.T * scale)
        size = torch.where(p[h] > 0, size, torch.zeros_like(size)).amax(-1, keepdim=True)
        rel = 2 * (2 if tensor_cores else 1) * (hd + 4) * U32 * size * 1.5 + (n + 20) * U32
        if outliers:
            rel = rel + 2 * 2.0 ** -18 * q[:rows, h].double().abs().amax(-1, keepdim=True) * kk.sum(-1).amax() * scale
        if tensor_cores:
            rel = rel + 2.0 ** -8
        tol[:, h] = rel * (p[h].nan_to_num(0) @ vv)
        if tensor_cores and vs is not None:
            peak = (p[h].nan_to_num(0) * vs[h // group, :n].double().nan_to_num(0)).amax(-1, keepdim=True)
            tol[:, h] += 2.0 ** -17 * peak * v8[h // group, :n].double().nan_to_num(0).abs().sum(0)
    return tol * 1.01 + HALF[dtype] * o.abs()

"""The operators around a K / V cache (include/depcap.h, "operators around a K / V cache") on torch tensors.

A layer of a caller who drives the backbone himself: `qk_norm_rope` on the projections, `cache_write` of the rows'
keys and values behind the context, `tree_attention` of the queries over the cache.  `cache_read` gives an 8-bit cache
back as the arrays that `DepCap.step` takes.  Like the rest of the binding this marshals arguments only; work goes to
`stream`, by default the current stream of the tensors' device."""
from __future__ import annotations

import ctypes as C

import torch

from . import binding as _b

_TYPES = {torch.float32: _b.DC_F32, torch.bfloat16: _b.DC_BF16, torch.float8_e4m3fn: _b.DC_E4M3}
_I64x2, _I64x3, _I64x5 = C.c_int64 * 2, C.c_int64 * 3, C.c_int64 * 5


class _Lengths:
    """A host array of int32 for the length of a call: a CPU int32 tensor as it is, anything else copied."""

    def __init__(self, values, batch, what):
        if isinstance(values, torch.Tensor) and values.dtype == torch.int32 and not values.is_cuda and values.is_contiguous():
            self.n, self.at, self.keep = values.numel(), values.data_ptr(), values
        else:
            values = values.tolist() if isinstance(values, torch.Tensor) else [int(v) for v in values]
            if any(not -2 ** 31 <= v < 2 ** 31 for v in values):
                raise ValueError(f"{what}: a value is outside 32 bits")
            self.n, self.keep = len(values), (C.c_int32 * max(len(values), 1))(*values)
            self.at = C.addressof(self.keep)
        if self.n != batch:
            raise ValueError(f"{what} has {self.n} lengths for {batch} sequences")


def _type(t, what):
    try:
        return _TYPES[t.dtype]
    except KeyError:
        raise TypeError(f"{what} is {t.dtype}: float32, bfloat16 or (a cache) float8_e4m3fn is wanted") from None


def _on(device, *tensors):
    for t in tensors:
        if t is not None and t.device != device:
            raise ValueError(f"a tensor is on {t.device}, another on {device}")


def _apart(t, what):
    """Whether a tensor that is written has a place of its own for every value (expanded ones have not)."""
    for n, s in zip(t.shape, t.stride()):
        if n > 1 and s == 0:
            raise ValueError(f"{what} is written: an expanded tensor has one place for several values")


def _run(call, device, stream, *args):
    if device.type != "cuda":
        raise RuntimeError("the operators need tensors on a CUDA device; there is no CPU path")
    if device.index == torch.cuda.current_device():
        rc = call(*args, (stream or torch.cuda.current_stream(device)).cuda_stream)
    else:
        with torch.cuda.device(device):
            rc = call(*args, (stream or torch.cuda.current_stream(device)).cuda_stream)
    if rc != _b.DC_OK:
        raise _b.DepCapError(rc, _b.lib().dc_last_error(None).decode())


class KvCache:
    """K and V of every layer: k [layers, slots, kv heads, keys, head_dim], v [layers, slots, kv heads, head_dim, keys],
    contiguous, in fp32 or bf16 (then the arrays that `DepCap.step` takes) or in float8_e4m3fn with one fp32 scale per key
    and kv head, k_scale and v_scale [layers, slots, kv heads, keys]."""

    def __init__(self, k, v, k_scale=None, v_scale=None):
        if k.dim() != 5 or tuple(v.shape) != tuple(k.shape[:3]) + (k.shape[4], k.shape[3]) or v.dtype != k.dtype:
            raise ValueError(f"k {tuple(k.shape)} {k.dtype} and v {tuple(v.shape)} {v.dtype} are not K and transposed V of one cache")
        if (k.dtype == torch.float8_e4m3fn) != (k_scale is not None) or (k_scale is None) != (v_scale is None):
            raise ValueError("an e4m3 cache has scales of K and of V, another none")
        for s in (k_scale, v_scale):
            if s is not None and (s.shape != k.shape[:4] or s.dtype != torch.float32):
                raise ValueError(f"scales are float32 {tuple(k.shape[:4])}")
        if not all(t is None or t.is_contiguous() for t in (k, v, k_scale, v_scale)):
            raise ValueError("the arrays of a cache are contiguous")
        _on(k.device, v, k_scale, v_scale)
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.n_layers, self.max_batch, self.n_kv_heads, self.max_ctx, self.head_dim = k.shape
        self.dtype, self.device = k.dtype, k.device
        self._c = _b.dc_cache(_type(k, "a cache"), *k.shape, k.data_ptr(), v.data_ptr(),
                              None if k_scale is None else k_scale.data_ptr(), None if v_scale is None else v_scale.data_ptr())
        self._ref = C.byref(self._c)

    @classmethod
    def empty(cls, n_layers, max_batch, n_kv_heads, max_ctx, head_dim, dtype=torch.float8_e4m3fn, device="cuda"):
        """A cache without keys (zeros)."""
        new = lambda *shape, dtype: torch.zeros(shape, dtype=dtype, device=device)
        scales = [new(n_layers, max_batch, n_kv_heads, max_ctx, dtype=torch.float32) if dtype == torch.float8_e4m3fn else None
                  for _ in range(2)]
        return cls(new(n_layers, max_batch, n_kv_heads, max_ctx, head_dim, dtype=dtype),
                   new(n_layers, max_batch, n_kv_heads, head_dim, max_ctx, dtype=dtype), *scales)

    def rows(self):
        """K and V as `cache_write` and `cache_read` see rows, views [layer, sequence, row, kv head, dim] of a cache that is not
        in 8 bits: a context of `DepCap.step` is written into an 8-bit cache, or read into, with these."""
        return self.k.transpose(2, 3), self.v.permute(0, 1, 4, 2, 3)


def _rows(cache, k, v, pos, n, layer):
    if k.dim() == 4:
        k = k[None]
    if v.dim() == 4:
        v = v[None]
    if k.dim() != 5 or k.shape != v.shape or k.dtype != v.dtype:
        raise ValueError(f"k {tuple(k.shape)} {k.dtype} and v {tuple(v.shape)} {v.dtype}: [layer,] sequence, row, kv head, dim of one type")
    layers, batch, most, heads, hd = k.shape
    if heads != cache.n_kv_heads or hd != cache.head_dim:
        raise ValueError(f"rows of {heads} x {hd} with a cache of {cache.n_kv_heads} x {cache.head_dim}")
    _on(cache.device, k, v)
    pos, n = _Lengths(pos, batch, "pos"), _Lengths([most] * batch if n is None else n, batch, "n")
    for i in range(batch):
        if C.c_int32.from_address(n.at + 4 * i).value > most:
            raise ValueError(f"n[{i}] is more than the {most} rows given")
    r = _b.dc_cache_rows(batch, layer, layers, _type(k, "rows"), k.data_ptr(), v.data_ptr(), _I64x5(*k.stride()),
                         _I64x5(*v.stride()), pos.at, n.at)
    return r, (pos, n)


def cache_write(cache, k, v, pos, n=None, layer=0, stream=None):
    """dc_cache_write: rows k, v [layers, sequences, rows, kv heads, head_dim] (or without the layers: one) become keys
    pos[b] .. pos[b] + n[b] - 1 of slot b in the cache's layers from `layer` on.  Any strides; n: all rows."""
    r, keep = _rows(cache, k, v, pos, n, layer)
    _run(_b.lib().dc_cache_write, cache.device, stream, cache._ref, C.byref(r))
    return cache


def cache_read(cache, k, v, pos, n=None, layer=0, stream=None):
    """dc_cache_read: the other way round, into k and v; rows >= n[b] are left as they were."""
    _apart(k, "k")
    _apart(v, "v")
    r, keep = _rows(cache, k, v, pos, n, layer)
    _run(_b.lib().dc_cache_read, cache.device, stream, cache._ref, C.byref(r))
    return k, v


def qk_norm_rope(q, k, pos, q_gain=None, k_gain=None, eps=1e-5, rope_theta=10000.0, q_out=None, k_out=None, stream=None):
    """dc_qk_norm_rope: q [rows, q heads, head_dim], k [rows, kv heads, head_dim] (contiguous dims, else any strides), pos
    int32 [rows] on the device, gains [head_dim] of q's type (None: 1).  Returns q_out, k_out (new ones where None; they may
    be q and k themselves)."""
    if q.dim() != 3 or k.dim() != 3 or q.shape[0] != k.shape[0] or q.shape[2] != k.shape[2] or q.dtype != k.dtype:
        raise ValueError(f"q {tuple(q.shape)} {q.dtype}, k {tuple(k.shape)} {k.dtype}: [rows, heads, head_dim] of one type")
    if q_out is None:
        q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    if k_out is None:
        k_out = torch.empty(k.shape, dtype=k.dtype, device=k.device)
    rows, hq, hd = q.shape
    if q_out.shape != q.shape or k_out.shape != k.shape or q_out.dtype != q.dtype or k_out.dtype != q.dtype:
        raise ValueError("an output has another shape or type than its input")
    if pos.shape != (rows,) or pos.dtype != torch.int32 or not pos.is_contiguous():
        raise ValueError(f"pos is a contiguous int32 tensor of {rows} positions")
    for g in (q_gain, k_gain):
        if g is not None and (g.shape != (hd,) or g.dtype != q.dtype or not g.is_contiguous()):
            raise ValueError(f"a gain is a contiguous tensor of {hd} values of {q.dtype}")
    qs, ks, qos, kos = q.stride(), k.stride(), q_out.stride(), k_out.stride()
    if hd > 1 and not qs[2] == ks[2] == qos[2] == kos[2] == 1:
        raise ValueError("the dims of a head are contiguous")
    _on(q.device, k, pos, q_gain, k_gain, q_out, k_out)
    for x, y in ((q, q_out), (k, k_out)):
        _apart(y, "an output")
        if x.numel() and x.data_ptr() == y.data_ptr() and x.stride() != y.stride():
            raise ValueError("an output in the place of its input has the same strides")
    a = _b.dc_qk_in(_type(q, "q"), rows, hq, k.shape[1], hd, eps, rope_theta, q.data_ptr(), k.data_ptr(), _I64x2(qs[0], qs[1]),
                    _I64x2(ks[0], ks[1]), None if q_gain is None else q_gain.data_ptr(),
                    None if k_gain is None else k_gain.data_ptr(), pos.data_ptr(), q_out.data_ptr(), k_out.data_ptr(),
                    _I64x2(qos[0], qos[1]), _I64x2(kos[0], kos[1]))
    _run(_b.lib().dc_qk_norm_rope, q.device, stream, C.byref(a))
    return q_out, k_out


def tree_attention(q, cache, ctx_len, n_rows, mask=None, layer=0, scale=None, out=None, workspace=None, status=None, stream=None):
    """dc_tree_attention: q [sequences, rows, q heads, head_dim] over slot b's first ctx_len[b] keys and, by the mask, the
    n_rows[b] drafted ones behind them.  mask int32 [sequences, rows, (rows + 31) // 32] on the device (`tree_mask`); None: all
    rows of a sequence see one another.  Returns out, like q; its rows >= n_rows[b] are left as they were (zeros in a new one).
    workspace: a uint8 tensor on the device for callers that keep one (`tree_attention_workspace` bytes)."""
    if q.dim() != 4 or q.shape[3] != cache.head_dim:
        raise ValueError(f"q {tuple(q.shape)}: sequences, rows, heads, head_dim={cache.head_dim}")
    batch, rows, heads, hd = q.shape
    if out is None:
        out = torch.zeros(q.shape, dtype=q.dtype, device=q.device)
    elif out.shape != q.shape or out.dtype != q.dtype:
        raise ValueError("out has another shape or type than q")
    if q.stride(3) != 1 or out.stride(3) != 1:
        raise ValueError("the dims of a head are contiguous")
    _apart(out, "out")
    if mask is not None and (mask.shape != (batch, rows, (rows + 31) // 32) or mask.dtype not in (torch.int32, torch.uint32)
                             or not mask.is_contiguous()):
        raise ValueError(f"the mask is a contiguous int32 tensor {(batch, rows, (rows + 31) // 32)}")
    if status is not None and (status.dtype != torch.int32 or status.numel() != 1):
        raise ValueError("status is one int32")
    if scale is not None and not scale > 0:
        raise ValueError("scale must be positive")
    _on(cache.device, q, out, mask, workspace, status)
    ctx, n = _Lengths(ctx_len, batch, "ctx_len"), _Lengths(n_rows, batch, "n_rows")
    qs, os_ = q.stride(), out.stride()
    a = _b.dc_tree_in(batch, layer, _type(q, "q"), heads, rows, scale or 0.0, q.data_ptr(), out.data_ptr(), _I64x3(*qs[:3]),
                      _I64x3(*os_[:3]), ctx.at, n.at, None if mask is None else mask.data_ptr(), None, 0,
                      None if status is None else status.data_ptr())
    if workspace is None:
        need = _need(cache, a)
        if need:
            # (of the stream that the work goes to, so that the allocator hands it out again in that order)
            if stream is None:
                workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
            else:
                with torch.cuda.stream(stream):
                    workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
    if workspace is not None:
        a.workspace, a.workspace_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    _run(_b.lib().dc_tree_attention, cache.device, stream, cache._ref, C.byref(a))
    return out


def _need(cache, a):
    if cache.device.type != "cuda":
        raise RuntimeError("the operators need tensors on a CUDA device; there is no CPU path")
    need = C.c_uint64()
    if cache.device.index == torch.cuda.current_device():
        rc = _b.lib().dc_tree_attention_workspace(cache._ref, C.byref(a), C.byref(need))
    else:
        with torch.cuda.device(cache.device):
            rc = _b.lib().dc_tree_attention_workspace(cache._ref, C.byref(a), C.byref(need))
    if rc != _b.DC_OK:
        raise _b.DepCapError(rc, _b.lib().dc_last_error(None).decode())
    return need.value


def tree_attention_workspace(q, cache, ctx_len, n_rows):
    """Bytes that tree_attention wants of a workspace for these lengths."""
    batch, rows, heads, hd = q.shape
    ctx, n = _Lengths(ctx_len, batch, "ctx_len"), _Lengths(n_rows, batch, "n_rows")
    a = _b.dc_tree_in(batch=batch, layer=0, dtype=_type(q, "q"), n_q_heads=heads, max_rows=rows, q=q.data_ptr(), o=q.data_ptr(),
                      q_stride=_I64x3(*q.stride()[:3]), o_stride=_I64x3(*q.stride()[:3]), ctx_len=ctx.at, n_rows=n.at)
    return _need(cache, a)


def tree_mask(parents, rows=None):
    """dc_tree_mask for a batch, on the host: parents [sequences][rows], each an earlier row or -1 -> int32 tensor
    [sequences, rows, (rows + 31) // 32] (pinned memory is the caller's business)."""
    rows = max((len(p) for p in parents), default=0) if rows is None else rows
    words = (rows + 31) // 32
    mask = torch.zeros((len(parents), rows, words), dtype=torch.int32)
    for b, p in enumerate(parents):
        if len(p) > rows:
            raise ValueError(f"sequence {b} has {len(p)} rows, more than {rows}")
        rc = _b.lib().dc_tree_mask((C.c_int32 * max(len(p), 1))(*[int(x) for x in p]), len(p), words, mask[b].data_ptr())
        if rc != _b.DC_OK:
            raise _b.DepCapError(rc, _b.lib().dc_last_error(None).decode())
    return mask

"""The operators around a K / V cache (include/depcap.h, "operators around a K / V cache") on torch tensors.

A layer of a caller who drives the backbone himself: `qk_norm_rope` on the projections, `cache_write` of the rows'
keys and values behind the context, `tree_attention` of the queries over the cache.  `cache_read` gives an 8-bit cache
back as the arrays that `DepCap.step` takes.  Like the rest of the binding this marshals arguments only; work goes to
`stream`, by default the current stream of the tensors' device.

For one token the calls cost more host time than device time, so the structures of the C calls are packed as bytes
(the layouts of binding.dc_cache .. dc_tree_in, which the tests compare)."""
from __future__ import annotations

import ctypes as C
from array import array
from contextlib import nullcontext
from struct import Struct

import torch

from . import binding as _b

_TYPES = {torch.float32: _b.DC_F32, torch.bfloat16: _b.DC_BF16, torch.float8_e4m3fn: _b.DC_E4M3}
_CACHE, _ROWS = Struct("@6i4P"), Struct("@4i2P10q2P")
_QK, _TREE = Struct("@5i2f2P4q5P4q"), Struct("@5if2P6q4PQP")
_Tensor, _INT32 = torch.Tensor, torch.int32


def _type(t, what):
    try:
        return _TYPES[t.dtype]
    except KeyError:
        raise TypeError(f"{what} is {t.dtype}: float32, bfloat16 or (a cache) float8_e4m3fn is wanted") from None


def _lengths(values, batch, what):
    """(address, owner) of a host array of `batch` int32: a CPU int32 tensor as it is, anything else copied"""
    if type(values) is _Tensor:
        if values.dtype is _INT32 and not values.is_cuda and values.is_contiguous():
            if values.numel() != batch:
                raise ValueError(f"{what} has {values.numel()} lengths for {batch} sequences")
            return values.data_ptr(), values
        values = values.tolist()
    try:
        held = array("i", [int(v) for v in values])
    except OverflowError:
        raise ValueError(f"{what}: a value is outside 32 bits") from None
    if len(held) != batch:
        raise ValueError(f"{what} has {len(held)} lengths for {batch} sequences")
    return held.buffer_info()[0], held


def _apart(shape, stride, what):
    """A tensor that is written has a place of its own for every value (an expanded one has not)."""
    if 0 in stride:
        for n, s in zip(shape, stride):
            if n > 1 and s == 0:
                raise ValueError(f"{what} is written: an expanded tensor has one place for several values")


def _elsewhere(device, *tensors):
    for t in tensors:
        if t is not None and t.device != device:
            raise ValueError(f"a tensor is on {t.device}, another on {device}")


def _on_cuda(index):
    if index < 0:
        raise RuntimeError("the operators need tensors on a CUDA device; there is no CPU path")


# (a torch without CUDA has neither)
_current, _stream_of = (getattr(torch._C, n, None) for n in ("_cuda_getDevice", "_cuda_getCurrentRawStream"))


def _call(f, index, stream, *args):
    """f(*args, stream) with device `index` current (-1: not a CUDA device)"""
    if index < 0:
        _on_cuda(index)
    if stream is None:
        raw = _stream_of(index)
    else:
        if stream.device_index != index:
            raise ValueError(f"a stream of device {stream.device_index} for tensors of device {index}")
        raw = stream.cuda_stream
    if index == _current():
        rc = f(*args, raw)
    else:
        with torch.cuda.device(index):
            rc = f(*args, raw)
    if rc != _b.DC_OK:
        raise _b.DepCapError(rc, _b.lib().dc_last_error(None).decode())


_HERE = nullcontext()


def _on(stream):
    """What is allocated (and filled) for a call belongs to the stream that its work goes to."""
    return _HERE if stream is None else torch.cuda.stream(stream)


class _Fn:
    """The library's functions, looked up once."""

    def __getattr__(self, name):
        f = getattr(_b.lib(), name)
        setattr(self, name, f)
        return f


_fn = _Fn()


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
        _elsewhere(k.device, v, k_scale, v_scale)
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.n_layers, self.max_batch, self.n_kv_heads, self.max_ctx, self.head_dim = k.shape
        self.dtype, self.device, self._index = k.dtype, k.device, k.get_device()
        self._c = _CACHE.pack(_type(k, "a cache"), *k.shape, k.data_ptr(), v.data_ptr(),
                              0 if k_scale is None else k_scale.data_ptr(), 0 if v_scale is None else v_scale.data_ptr())

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


def _move(f, cache, k, v, pos, n, layer, stream):
    shape, dtype = k.shape, k.dtype
    if len(shape) == 4:
        k, shape = k[None], (1, *shape)
    if v.dim() == 4:
        v = v[None]
    if v.shape != shape or v.dtype is not dtype or len(shape) != 5:
        raise ValueError(f"k {tuple(shape)} {dtype} and v {tuple(v.shape)} {v.dtype}: [layer,] sequence, row, kv head, dim of one type")
    layers, batch, most, heads, hd = shape
    if heads != cache.n_kv_heads or hd != cache.head_dim:
        raise ValueError(f"rows of {heads} x {hd} with a cache of {cache.n_kv_heads} x {cache.head_dim}")
    index = cache._index
    if k.get_device() != index or v.get_device() != index:
        _elsewhere(cache.device, k, v)
    at, keep = _lengths(pos, batch, "pos")
    n_at, n_keep = _lengths([most] * batch if n is None else n, batch, "n")
    if n is not None and max(n_keep.tolist(), default=0) > most:
        raise ValueError(f"n asks for more than the {most} rows given")
    if 0 in (layers, batch, most):       # nothing to do, and an empty tensor has no address
        return _on_cuda(index)
    _call(f, index, stream, cache._c, _ROWS.pack(batch, layer, layers, _type(k, "rows"), k.data_ptr(), v.data_ptr(), *k.stride(),
                                                 *v.stride(), at, n_at))


def cache_write(cache, k, v, pos, n=None, layer=0, stream=None):
    """dc_cache_write: rows k, v [layers, sequences, rows, kv heads, head_dim] (or without the layers: one) become keys
    pos[b] .. pos[b] + n[b] - 1 of slot b in the cache's layers from `layer` on.  Any strides; n: all rows."""
    _move(_fn.dc_cache_write, cache, k, v, pos, n, layer, stream)
    return cache


def cache_read(cache, k, v, pos, n=None, layer=0, stream=None):
    """dc_cache_read: the other way round, into k and v; rows >= n[b] are left as they were."""
    _apart(k.shape, k.stride(), "k")
    _apart(v.shape, v.stride(), "v")
    _move(_fn.dc_cache_read, cache, k, v, pos, n, layer, stream)
    return k, v


def qk_norm_rope(q, k, pos, q_gain=None, k_gain=None, eps=1e-5, rope_theta=10000.0, q_out=None, k_out=None, stream=None):
    """dc_qk_norm_rope: q [rows, q heads, head_dim], k [rows, kv heads, head_dim] (contiguous dims, else any strides), pos
    int32 [rows] on the device, gains [head_dim] of q's type (None: 1).  Returns q_out, k_out (new ones where None; they may
    be q and k themselves)."""
    dtype, index, shape, kshape = q.dtype, q.get_device(), q.shape, k.shape
    if len(shape) != 3 or len(kshape) != 3 or shape[0] != kshape[0] or shape[2] != kshape[2] or k.dtype is not dtype:
        raise ValueError(f"q {tuple(shape)} {dtype}, k {tuple(kshape)} {k.dtype}: [rows, heads, head_dim] of one type")
    rows, hq, hd = shape
    if q_out is None or k_out is None:
        with _on(stream):
            q_out = torch.empty(shape, dtype=dtype, device=q.device) if q_out is None else q_out
            k_out = torch.empty(kshape, dtype=dtype, device=q.device) if k_out is None else k_out
    if q_out.shape != shape or k_out.shape != kshape or q_out.dtype is not dtype or k_out.dtype is not dtype:
        raise ValueError("an output has another shape or type than its input")
    if pos.dtype is not _INT32 or pos.dim() != 1 or pos.numel() != rows or not pos.is_contiguous():
        raise ValueError(f"pos is a contiguous int32 tensor of {rows} positions")
    gain_at = [0, 0]
    for i, g in enumerate((q_gain, k_gain)):
        if g is not None:
            if g.dtype is not dtype or g.shape != (hd,) or not g.is_contiguous() or g.get_device() != index:
                raise ValueError(f"a gain is a contiguous tensor of {hd} values of {dtype} on {q.device}")
            gain_at[i] = g.data_ptr()
    if not k.get_device() == pos.get_device() == q_out.get_device() == k_out.get_device() == index:
        _elsewhere(q.device, k, pos, q_out, k_out)
    a, b, d = q.stride()
    e, f, h = k.stride()
    qo, ko = q_out.stride(), k_out.stride()
    if hd > 1 and not d == h == qo[2] == ko[2] == 1:
        raise ValueError("the dims of a head are contiguous")
    if 0 in qo or 0 in ko:
        _apart(shape, qo, "q_out")
        _apart(kshape, ko, "k_out")
    x, y, u, w = q.data_ptr(), k.data_ptr(), q_out.data_ptr(), k_out.data_ptr()
    if (x == u and x and qo != (a, b, d)) or (y == w and y and ko != (e, f, h)):
        raise ValueError("an output in the place of its input has the same strides")
    _call(_fn.dc_qk_norm_rope, index, stream,
          _QK.pack(_type(q, "q"), rows, hq, kshape[1], hd, eps, rope_theta, x, y, a, b, e, f, *gain_at, pos.data_ptr(), u, w, qo[0], qo[1],
                   ko[0], ko[1]))
    return q_out, k_out


def tree_attention(q, cache, ctx_len, n_rows, mask=None, layer=0, scale=None, out=None, workspace=None, status=None, stream=None):
    """dc_tree_attention: q [sequences, rows, q heads, head_dim] over slot b's first ctx_len[b] keys and, by the mask, the
    n_rows[b] drafted ones behind them.  mask int32 [sequences, rows, (rows + 31) // 32] on the device (`tree_mask`); None: all
    rows of a sequence see one another.  Returns out, like q, or q itself; its rows >= n_rows[b] are left as they were (zeros in a new one).
    workspace: a uint8 tensor on the device for callers that keep one (`tree_attention_workspace` bytes)."""
    shape, dtype, index = q.shape, q.dtype, cache._index
    if len(shape) != 4 or shape[3] != cache.head_dim:
        raise ValueError(f"q {tuple(shape)}: sequences, rows, heads, head_dim={cache.head_dim}")
    batch, rows, heads, hd = shape
    if out is None:
        with _on(stream):
            out = torch.zeros(shape, dtype=dtype, device=q.device)
    elif out.shape != shape or out.dtype != dtype:
        raise ValueError("out has another shape or type than q")
    a, b, h, d = q.stride()
    os_ = out.stride()
    if d != 1 or os_[3] != 1:
        raise ValueError("the dims of a head are contiguous")
    if 0 in os_:
        _apart(shape, os_, "out")
    if os_ != (a, b, h, d) and out.data_ptr() == q.data_ptr() and any(m > 1 and x != y for m, x, y in zip(shape, os_, (a, b, h, d))):
        raise ValueError("an output in the place of its input has the same strides")
    mask_at = 0
    if mask is not None:
        if mask.dtype not in (torch.int32, torch.uint32) or mask.shape != (batch, rows, (rows + 31) // 32) or not mask.is_contiguous():
            raise ValueError(f"the mask is a contiguous int32 tensor {(batch, rows, (rows + 31) // 32)}")
        mask_at = mask.data_ptr()
    if status is not None and (status.dtype != torch.int32 or status.numel() != 1):
        raise ValueError("status is one int32")
    if workspace is not None and not workspace.is_contiguous():
        raise ValueError("the workspace is contiguous")
    if scale is None:
        scale = 0.0
    elif not scale >= 2.0 ** -126:        # (what fp32 rounds to 0 would be the default)
        raise ValueError("scale must be positive, a normal fp32 number")
    if q.get_device() != index or out.get_device() != index or workspace is not None or status is not None or \
            (mask is not None and mask.get_device() != index):
        _elsewhere(cache.device, q, out, mask, workspace, status)
    ctx, keep = _lengths(ctx_len, batch, "ctx_len")
    n, n_keep = _lengths(n_rows, batch, "n_rows")
    if batch == 0 or rows == 0:
        _on_cuda(index)
        return out
    args = (batch, layer, _type(q, "q"), heads, rows, scale, q.data_ptr(), out.data_ptr(), a, b, h, os_[0], os_[1], os_[2], ctx, n, mask_at)
    st = 0 if status is None else status.data_ptr()
    call = _fn.dc_tree_attention
    if workspace is None:
        # most calls want none: whether this one does is asked only after a refusal, which launches nothing
        try:
            _call(call, index, stream, cache._c, _TREE.pack(*args, 0, 0, st))
            return out
        except _b.DepCapError:
            size = _need(cache, _TREE.pack(*args, 0, 0, st))
            if not size:
                raise
        with _on(stream):
            workspace = torch.empty(size, dtype=torch.uint8, device=cache.device)
    _call(call, index, stream, cache._c, _TREE.pack(*args, workspace.data_ptr(), workspace.numel() * workspace.element_size(), st))
    return out


def _need(cache, packed):
    need = C.c_uint64()
    _call(lambda c, a, stream: _fn.dc_tree_attention_workspace(c, a, C.addressof(need)), cache._index, None, cache._c, packed)
    return need.value


def tree_attention_workspace(q, cache, ctx_len, n_rows):
    """Bytes that tree_attention wants of a workspace for these lengths."""
    batch, rows, heads, hd = q.shape
    ctx, keep = _lengths(ctx_len, batch, "ctx_len")
    n, n_keep = _lengths(n_rows, batch, "n_rows")
    if batch == 0 or rows == 0:
        return 0
    s = q.stride()
    return _need(cache, _TREE.pack(batch, 0, _type(q, "q"), heads, rows, 0.0, q.data_ptr(), q.data_ptr(), s[0], s[1], s[2], s[0], s[1], s[2],
                                   ctx, n, 0, 0, 0, 0))


def tree_mask(parents, rows=None):
    """dc_tree_mask for a batch, on the host: parents [sequences][rows], each an earlier row or -1 -> int32 tensor
    [sequences, rows, (rows + 31) // 32]."""
    rows = max((len(p) for p in parents), default=0) if rows is None else rows
    words = (rows + 31) // 32
    mask = torch.zeros((len(parents), rows, words), dtype=torch.int32)
    for b, p in enumerate(parents):
        if len(p) > rows:
            raise ValueError(f"sequence {b} has {len(p)} rows, more than {rows}")
        try:
            parent = array("i", [int(x) for x in p] or [-1])
        except OverflowError:
            raise ValueError(f"sequence {b}: a parent is outside 32 bits") from None
        rc = _b.lib().dc_tree_mask(C.cast(parent.buffer_info()[0], _b._I32P), len(p), words, mask[b].data_ptr())
        if rc != _b.DC_OK:
            raise _b.DepCapError(rc, _b.lib().dc_last_error(None).decode())
    return mask

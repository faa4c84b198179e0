// dc_cache_write / dc_cache_read: rows of K and V into a cache and back, in 8 bits or as they are.
#include "ops.h"
#include "pdl.cuh"

namespace dc {
namespace {

struct RowsArgs {
  dc_cache c;
  char *k, *v;
  long long ks[5], vs[5];
  int layer, pos[DC_MAX_BATCH], n[DC_MAX_BATCH];
};

// ---- any strides, types and alignment: a warp takes one row of K or V -----------------------------------
// (32 layers of four contexts of up to 1024 keys 6353 us, 13 times k_rows_tile: V goes out value by value.  V with contiguous keys comes
// here, K with it, where a first position is no multiple of 16 bytes: its pieces would lie across the cache's)
// grid (row, sequence * kv head, layer * 2 + side)
constexpr int kAnyWarps = 8;

template <typename T, typename H, bool WRITE>
__global__ void __launch_bounds__(kAnyWarps * 32) k_rows_any(const RowsArgs a) {
  pdl_trigger();
  pdl_wait();
  const int lane = threadIdx.x & 31, nkv = a.c.n_kv_heads, hd = a.c.head_dim;
  const int b = blockIdx.y / nkv, g = blockIdx.y % nkv, side = blockIdx.z & 1, l = blockIdx.z >> 1;
  const long long* st = side ? a.vs : a.ks;
  T* rows = reinterpret_cast<T*>(side ? a.v : a.k) + l * st[0] + b * st[1] + g * st[3];
  const size_t slot = ((size_t)(a.layer + l) * a.c.max_batch + b) * nkv + g;
  H* held = reinterpret_cast<H*>(side ? a.c.v : a.c.k) + slot * a.c.max_ctx * hd;
  float* scales = side ? a.c.v_scale : a.c.k_scale;
  const size_t kstep = side ? 1 : hd, dstep = side ? a.c.max_ctx : 1;
  constexpr bool Q = sizeof(H) == 1;
  for (int r = blockIdx.x * kAnyWarps + (threadIdx.x >> 5); r < a.n[b]; r += gridDim.x * kAnyWarps) {
    T* row = rows + r * st[2];
    const int key = a.pos[b] + r;
    H* h = held + key * kstep;
    if (WRITE) {
      float x[8], top = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int d = i * 32 + lane;
        x[i] = d < hd ? op_f32(row[d * st[4]]) : 0.f;
        top = fmaxf(top, op_magnitude(x[i]));
      }
      float inv = 1.f;
      if (Q) {
#pragma unroll
        for (int s = 16; s >= 1; s >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, s));
        const float sc = op_scale(top);
        inv = __fdiv_rn(1.f, sc);
        if (lane == 0) scales[slot * a.c.max_ctx + key] = sc;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int d = i * 32 + lane;
        if (d < hd) {
          if constexpr (Q) h[d * dstep].__x = __nv_cvt_float_to_fp8(x[i] * inv, __NV_SATFINITE, __NV_E4M3);
          else h[d * dstep] = op_to<H>(x[i]);
        }
      }
    } else {
      const float sc = Q ? scales[slot * a.c.max_ctx + key] : 1.f;
      for (int d = lane; d < hd; d += 32) row[d * st[4]] = op_to<T>(Q ? op_f32(h[d * dstep]) * sc : op_f32(h[d * dstep]));
    }
  }
}

// ---- rows that move in 16-byte pieces, head_dim 64 or 128 ----------------------------------------------
// grid (tile, sequence * kv head, layer * 2 + side): a CTA takes K or V of 64 keys.  Tiles start at multiples of 64 keys, so
// that only the first and the last of a sequence write less than whole pieces of V^T.
//   K, either way: 16 (8) lanes a row, 8 dims a lane.
//   V with contiguous dims: the same, four keys a thread, whose values turn into groups of four keys in shared memory.
//   V with contiguous keys (ACROSS): 8 keys x 1 dim a lane; a row's maximum comes together over the CTA.
// Bound by HBM (2 bytes read for 1 written): 32 layers of four contexts of up to 1024 keys, 2.87 GB, 480 us (6.0 TB/s; 516 .. 534 where
// passes go on for a second) with contiguous keys, 543 us with contiguous dims (5.3); 28 layers of four contexts of 768 keys back, 267
// MB, 41 us (6.5), as rows 58 (4.6); 16 layers of a bf16 cache written 308 us (6.2), read as rows 378 (5.0).  Ordinary instructions for a value: one to unpack, one for the maximum (of 16-bit
// patterns, two at a time), a half to multiply, a half to convert.
constexpr int kTk = 64, kTileThreads = 256;

template <typename H> struct Four { static constexpr int bytes = 4 * sizeof(H); };   // a group of four keys

// largest magnitude of 8 values, as long as all are finite; else something above every finite one
template <typename T> struct Piece;            // 8 values as they come
template <> struct Piece<__nv_bfloat16> {
  uint4 w;
  __device__ __forceinline__ void load(const void* p) { w = *static_cast<const uint4*>(p); }
  __device__ __forceinline__ void store(void* p) const { *static_cast<uint4*>(p) = w; }
  __device__ __forceinline__ uint32_t word(int i) const { return i == 0 ? w.x : i == 1 ? w.y : i == 2 ? w.z : w.w; }
  __device__ __forceinline__ float at(int i) const { return __uint_as_float(i & 1 ? word(i >> 1) & 0xffff0000u : word(i >> 1) << 16); }
  __device__ __forceinline__ void set(int i, float x0, float x1) {      // values 2 i and 2 i + 1
    __nv_bfloat162 p = __floats2bfloat162_rn(x0, x1);
    const uint32_t u = *reinterpret_cast<uint32_t*>(&p);
    if (i == 0) w.x = u; else if (i == 1) w.y = u; else if (i == 2) w.z = u; else w.w = u;
  }
};
template <> struct Piece<float> {
  float4 w[2];
  __device__ __forceinline__ void load(const void* p) { w[0] = static_cast<const float4*>(p)[0]; w[1] = static_cast<const float4*>(p)[1]; }
  __device__ __forceinline__ void store(void* p) const { static_cast<float4*>(p)[0] = w[0]; static_cast<float4*>(p)[1] = w[1]; }
  __device__ __forceinline__ float at(int i) const { const float4& v = w[i >> 2]; return (i & 3) == 0 ? v.x : (i & 3) == 1 ? v.y : (i & 3) == 2 ? v.z : v.w; }
  __device__ __forceinline__ void set(int i, float x0, float x1) {
    float4& v = w[i >> 1];
    if (i & 1) { v.z = x0; v.w = x1; } else { v.x = x0; v.y = x1; }
  }
};
template <> struct Piece<__nv_fp8_e4m3> {
  uint2 w;
  __device__ __forceinline__ void load(const void* p) { w = *static_cast<const uint2*>(p); }
  __device__ __forceinline__ void store(void* p) const { *static_cast<uint2*>(p) = w; }
  __device__ __forceinline__ void pair(int i, float& x0, float& x1) const {
    const uint32_t u = i < 2 ? w.x : w.y;
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(i & 1 ? u >> 16 : u & 0xffffu), __NV_E4M3);
    const float2 f = __half22float2(__half2(h));
    x0 = f.x; x1 = f.y;
  }
};

__device__ __forceinline__ float piece_max(const Piece<__nv_bfloat16>& p) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) asm("max.u16x2 %0, %0, %1;" : "+r"(m) : "r"(p.word(i) & 0x7fff7fffu));
  return __uint_as_float(max(m & 0xffffu, m >> 16) << 16);    // (patterns order as magnitudes do, infinities and NaN on top)
}
__device__ __forceinline__ float piece_max(const Piece<float>& p) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(p.at(i)) & 0x7fffffffu);
  return __uint_as_float(m);
}
// largest magnitude of each of 8 keys over some dims, infinities and NaN on top
template <int D>
__device__ __forceinline__ void piece_max_keys(const Piece<__nv_bfloat16> (&p)[D], float (&top)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t m = 0;
#pragma unroll
    for (int d = 0; d < D; ++d) asm("max.u16x2 %0, %0, %1;" : "+r"(m) : "r"(p[d].word(i) & 0x7fff7fffu));
    top[2 * i] = __uint_as_float(m << 16);
    top[2 * i + 1] = __uint_as_float(m & 0xffff0000u);
  }
}
template <int D>
__device__ __forceinline__ void piece_max_keys(const Piece<float> (&p)[D], float (&top)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    uint32_t m = 0;
#pragma unroll
    for (int d = 0; d < D; ++d) m = max(m, __float_as_uint(p[d].at(e)) & 0x7fffffffu);
    top[e] = __uint_as_float(m);
  }
}
template <typename T>
__device__ __forceinline__ float piece_max_finite(const Piece<T>& p) {
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = fmaxf(m, op_magnitude(p.at(i)));
  return m;
}
__device__ __forceinline__ bool not_finite(float magnitude) { return !(magnitude <= 3.402823466e38f); }

// values 2 i, 2 i + 1 times inv as two e4m3 bytes
template <typename T>
__device__ __forceinline__ uint32_t quant2(const Piece<T>& p, int i, float inv) {
  return __nv_cvt_float2_to_fp8x2(make_float2(p.at(2 * i) * inv, p.at(2 * i + 1) * inv), __NV_SATFINITE, __NV_E4M3);
}

template <typename T, typename H, int HD, bool WRITE, bool ACROSS>
__global__ void __launch_bounds__(kTileThreads) k_rows_tile(const __grid_constant__ RowsArgs a) {
  constexpr bool Q = sizeof(H) == 1;
  constexpr int LPR = HD / 8;                     // lanes a row
  constexpr int RPT = kTk * LPR / kTileThreads;   // rows a thread: 4 (128), 2 (64)
  const int nkv = a.c.n_kv_heads, b = blockIdx.y / nkv, g = blockIdx.y % nkv, side = blockIdx.z & 1, l = blockIdx.z >> 1;
  const int pos = a.pos[b], end = pos + a.n[b], t0 = (pos / kTk + blockIdx.x) * kTk;
  pdl_wait();      // (no pdl_trigger: blocks of the next kernel in the places of these cost 5% of a large write)
  if (t0 >= end) return;
  const int lo = max(pos, t0), hi = min(end, t0 + kTk), tid = threadIdx.x;
  const long long* st = side ? a.vs : a.ks;
  T* rows = reinterpret_cast<T*>(side ? a.v : a.k) + l * st[0] + b * st[1] + g * st[3];
  const size_t slot = ((size_t)(a.layer + l) * a.c.max_batch + b) * nkv + g;
  H* held = reinterpret_cast<H*>(side ? a.c.v : a.c.k) + slot * a.c.max_ctx * HD;
  float* scales = Q ? (side ? a.c.v_scale : a.c.k_scale) + slot * a.c.max_ctx : nullptr;
  __shared__ __align__(16) char sh[ACROSS ? 8 * kTk * 4 + 16 : HD * (kTk / 4 + 1) * Four<H>::bytes];

  if (!ACROSS || side == 0) {
    const int c = tid % LPR, r0 = tid / LPR * RPT;    // dims 8 c .. + 7 of rows t0 + r0 .. + RPT - 1
    if (side == 0 || !ACROSS) {
      Piece<T> x[RPT];
      if (WRITE) {
#pragma unroll
        for (int j = 0; j < RPT; ++j) {
          const int key = t0 + r0 + j;
          if (key >= lo && key < hi) x[j].load(rows + (long long)(key - pos) * st[2] + c * 8);
          else x[j] = Piece<T>{};
        }
        Piece<H> y[RPT];
        if constexpr (Q) {
          float top[RPT];
#pragma unroll
          for (int j = 0; j < RPT; ++j) {
            top[j] = piece_max(x[j]);
            if (not_finite(top[j])) top[j] = piece_max_finite(x[j]);
#pragma unroll
            for (int s = LPR / 2; s >= 1; s >>= 1) top[j] = fmaxf(top[j], __shfl_xor_sync(0xffffffffu, top[j], s));
          }
          // lane c makes the scale of row c % RPT for the lanes of its rows (two divisions a lane and not two a row)
          float mine = top[0];
#pragma unroll
          for (int j = 1; j < RPT; ++j) mine = c % RPT == j ? top[j] : mine;
          const float sc = op_scale(mine), inv_mine = __fdiv_rn(1.f, sc);
          if (c < RPT && t0 + r0 + c >= lo && t0 + r0 + c < hi) scales[t0 + r0 + c] = sc;
#pragma unroll
          for (int j = 0; j < RPT; ++j) {
            const float inv = __shfl_sync(0xffffffffu, inv_mine, j, LPR);
            y[j].w.x = quant2(x[j], 0, inv) | quant2(x[j], 1, inv) << 16;
            y[j].w.y = quant2(x[j], 2, inv) | quant2(x[j], 3, inv) << 16;
          }
        } else {
#pragma unroll
          for (int j = 0; j < RPT; ++j) y[j] = x[j];
        }
        if (side == 0) {
#pragma unroll
          for (int j = 0; j < RPT; ++j) {
            const int key = t0 + r0 + j;
            if (key >= lo && key < hi) y[j].store(held + (size_t)key * HD + c * 8);
          }
          return;
        }
        // V: [dim][key] in shared memory, then out as groups of four keys
        H* tile = reinterpret_cast<H*>(sh);
        const H* yv = reinterpret_cast<const H*>(y);
#pragma unroll
        for (int d = 0; d < 8; ++d) {
          H* at = tile + (c * 8 + d) * (kTk + 4) + r0;
          if constexpr (Q) {
            uint32_t u = 0;
#pragma unroll
            for (int j = 0; j < RPT; ++j) u |= ((d < 4 ? y[j].w.x >> (8 * d) : y[j].w.y >> (8 * (d - 4))) & 0xffu) << (8 * j);
            if (RPT == 4) *reinterpret_cast<uint32_t*>(at) = u;
            else *reinterpret_cast<uint16_t*>(at) = (uint16_t)u;
          } else {
#pragma unroll
            for (int j = 0; j < RPT; ++j) at[j] = yv[j * 8 + d];
          }
        }
        __syncthreads();
        for (int i = tid; i < HD * kTk / 4; i += kTileThreads) {
          const int d = i / (kTk / 4), k4 = i % (kTk / 4) * 4, key = t0 + k4;
          const H* from = tile + d * (kTk + 4) + k4;
          H* to = held + (size_t)d * a.c.max_ctx + key;
          if (key >= lo && key + 4 <= hi) {
            if constexpr (sizeof(H) == 1) *reinterpret_cast<uint32_t*>(to) = *reinterpret_cast<const uint32_t*>(from);
            else if constexpr (sizeof(H) == 2) *reinterpret_cast<uint2*>(to) = *reinterpret_cast<const uint2*>(from);
            else *reinterpret_cast<uint4*>(to) = *reinterpret_cast<const uint4*>(from);
          } else {
            for (int e = 0; e < 4; ++e)
              if (key + e >= lo && key + e < hi) to[e] = from[e];
          }
        }
        return;
      }
      // ---- read ----
      Piece<H> y[RPT];
      if (side == 0) {
#pragma unroll
        for (int j = 0; j < RPT; ++j) {
          const int key = t0 + r0 + j;
          if (key >= lo && key < hi) y[j].load(held + (size_t)key * HD + c * 8);
        }
      } else {
        H* tile = reinterpret_cast<H*>(sh);
        for (int i = tid; i < HD * kTk / 4; i += kTileThreads) {    // (whole groups: the cache goes on to a multiple of 64 keys)
          const int d = i / (kTk / 4), k4 = i % (kTk / 4) * 4;
          H* to = tile + d * (kTk + 4) + k4;
          const H* from = held + (size_t)d * a.c.max_ctx + t0 + k4;
          if constexpr (sizeof(H) == 1) *reinterpret_cast<uint32_t*>(to) = *reinterpret_cast<const uint32_t*>(from);
          else if constexpr (sizeof(H) == 2) *reinterpret_cast<uint2*>(to) = *reinterpret_cast<const uint2*>(from);
          else *reinterpret_cast<uint4*>(to) = *reinterpret_cast<const uint4*>(from);
        }
        __syncthreads();
        H* yv = reinterpret_cast<H*>(y);
#pragma unroll
        for (int d = 0; d < 8; ++d) {
          const H* at = tile + (c * 8 + d) * (kTk + 4) + r0;
          if constexpr (Q) {
            const uint32_t u = RPT == 4 ? *reinterpret_cast<const uint32_t*>(at) : *reinterpret_cast<const uint16_t*>(at);
#pragma unroll
            for (int j = 0; j < RPT; ++j) {
              const uint32_t byte = ((u >> (8 * j)) & 0xffu) << (8 * (d & 3));
              if (d == 0) y[j].w.x = byte; else if (d == 4) y[j].w.y = byte; else if (d < 4) y[j].w.x |= byte; else y[j].w.y |= byte;
            }
          } else {
#pragma unroll
            for (int j = 0; j < RPT; ++j) yv[j * 8 + d] = at[j];
          }
        }
      }
#pragma unroll
      for (int j = 0; j < RPT; ++j) {
        const int key = t0 + r0 + j;
        if (key < lo || key >= hi) continue;
        if constexpr (Q) {
          const float sc = scales[key];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float x0, x1;
            y[j].pair(i, x0, x1);
            x[j].set(i, x0 * sc, x1 * sc);
          }
        } else {
          x[j] = y[j];
        }
        x[j].store(rows + (long long)(key - pos) * st[2] + c * 8);
      }
      return;
    }
  }

  if constexpr (ACROSS) {
    // V with contiguous keys on both sides: 8 keys a lane, dims d0, d0 + 32, ..
    constexpr int DPT = HD / 32;
    const int k8 = tid % 8 * 8, d0 = tid / 8, key = t0 + k8;
    const bool whole = key >= lo && key + 8 <= hi;
    if (!WRITE) {
      if (key >= hi || key + 8 <= lo) return;
      float sc[8];
      if constexpr (Q) {
        const float4 s0 = *reinterpret_cast<const float4*>(scales + key), s1 = *reinterpret_cast<const float4*>(scales + key + 4);
        sc[0] = s0.x; sc[1] = s0.y; sc[2] = s0.z; sc[3] = s0.w; sc[4] = s1.x; sc[5] = s1.y; sc[6] = s1.z; sc[7] = s1.w;
      }
      Piece<H> y[DPT];
#pragma unroll
      for (int i = 0; i < DPT; ++i) y[i].load(held + (size_t)(d0 + 32 * i) * a.c.max_ctx + key);
#pragma unroll
      for (int i = 0; i < DPT; ++i) {
        Piece<T> x;
        if constexpr (Q) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float x0, x1;
            y[i].pair(e, x0, x1);
            x.set(e, x0 * sc[2 * e], x1 * sc[2 * e + 1]);
          }
        } else {
          x = y[i];
        }
        T* to = rows + (d0 + 32 * i) * st[4] + (key - pos);
        if (whole) x.store(to);
        else
          for (int e = 0; e < 8; ++e)
            if (key + e >= lo && key + e < hi) to[e] = op_to<T>(x.at(e));
      }
      return;
    }
    Piece<T> x[DPT];
#pragma unroll
    for (int i = 0; i < DPT; ++i) {
      const T* from = rows + (d0 + 32 * i) * st[4] + (key - pos);
      if (whole) x[i].load(from);
      else {
        float f[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = key + e >= lo && key + e < hi ? op_f32(from[e]) : 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[i].set(e, f[2 * e], f[2 * e + 1]);
      }
    }
    if constexpr (Q) {
      float* part = reinterpret_cast<float*>(sh);    // [warp][key]
      float top[8];
      piece_max_keys(x, top);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (not_finite(top[e])) {
          top[e] = 0.f;
#pragma unroll
          for (int i = 0; i < DPT; ++i) top[e] = fmaxf(top[e], op_magnitude(x[i].at(e)));
        }
        top[e] = fmaxf(top[e], __shfl_xor_sync(0xffffffffu, top[e], 8));
        top[e] = fmaxf(top[e], __shfl_xor_sync(0xffffffffu, top[e], 16));
      }
      if ((tid & 31) < 8) {
#pragma unroll
        for (int e = 0; e < 8; ++e) part[(tid >> 5) * kTk + k8 + e] = top[e];
      }
      __syncthreads();
      if (tid < kTk) {    // a thread a key: the scale, and its reciprocal for everybody
        float m = 0.f;
#pragma unroll
        for (int w = 0; w < 8; ++w) m = fmaxf(m, part[w * kTk + tid]);
        const float sc = op_scale(m);
        if (t0 + tid >= lo && t0 + tid < hi) scales[t0 + tid] = sc;
        part[tid] = __fdiv_rn(1.f, sc);              // (read above by this thread alone)
      }
      __syncthreads();
      float inv[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) inv[e] = part[k8 + e];
#pragma unroll
      for (int i = 0; i < DPT; ++i) {
        uint32_t u[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
          u[e] = __nv_cvt_float2_to_fp8x2(make_float2(x[i].at(2 * e) * inv[2 * e], x[i].at(2 * e + 1) * inv[2 * e + 1]), __NV_SATFINITE, __NV_E4M3);
        Piece<H> y;
        y.w = make_uint2(u[0] | u[1] << 16, u[2] | u[3] << 16);
        H* to = held + (size_t)(d0 + 32 * i) * a.c.max_ctx + key;
        if (whole) y.store(to);
        else
          for (int e = 0; e < 8; ++e)
            if (key + e >= lo && key + e < hi) to[e].__x = (uint8_t)((e < 4 ? y.w.x >> (8 * e) : y.w.y >> (8 * (e - 4))) & 0xffu);
      }
    } else {
#pragma unroll
      for (int i = 0; i < DPT; ++i) {
        H* to = held + (size_t)(d0 + 32 * i) * a.c.max_ctx + key;
        if (whole) x[i].store(to);
        else
          for (int e = 0; e < 8; ++e)
            if (key + e >= lo && key + e < hi) to[e] = op_to<H>(x[i].at(e));
      }
    }
  }
}

template <typename T, typename H, bool WRITE>
void launch(const RowsArgs& a, int batch, int n_layers, int most, cudaStream_t s) {
  // 16-byte pieces: the rows', the cache's (its rows are 64 bytes at least)
  constexpr int e16 = 16 / sizeof(T);
  const int hd = a.c.head_dim;
  auto even = [](const long long* st, int from, int to) { bool ok = true; for (int i = from; i < to; ++i) ok = ok && st[i] % e16 == 0; return ok; };
  const bool base = op_aligned(a.k) && op_aligned(a.v) && op_aligned(a.c.k) && op_aligned(a.c.v) && op_aligned(a.c.k_scale) && op_aligned(a.c.v_scale);
  const bool k_ok = base && (hd == 64 || hd == 128) && a.ks[4] == 1 && even(a.ks, 0, 4);
  const bool v_rows = a.vs[4] == 1 && even(a.vs, 0, 4);
  bool v_across = a.vs[2] == 1 && even(a.vs, 0, 2) && even(a.vs, 3, 5);
  int tiles = 0;
  for (int b = 0; b < batch; ++b) {
    if (a.n[b] == 0) continue;
    v_across = v_across && a.pos[b] % e16 == 0;
    tiles = max(tiles, (a.pos[b] + a.n[b] + kTk - 1) / kTk - a.pos[b] / kTk);
  }
  if (k_ok && (v_rows || v_across)) {
    const dim3 grid(tiles, batch * a.c.n_kv_heads, 2 * n_layers);
    if (v_rows) {
      if (hd == 128) launch_chained(k_rows_tile<T, H, 128, WRITE, false>, grid, dim3(kTileThreads), 0, s, a);
      else launch_chained(k_rows_tile<T, H, 64, WRITE, false>, grid, dim3(kTileThreads), 0, s, a);
    } else {
      if (hd == 128) launch_chained(k_rows_tile<T, H, 128, WRITE, true>, grid, dim3(kTileThreads), 0, s, a);
      else launch_chained(k_rows_tile<T, H, 64, WRITE, true>, grid, dim3(kTileThreads), 0, s, a);
    }
    return;
  }
  // (rows beyond the grid are taken in further turns)
  const dim3 grid(min((most + kAnyWarps - 1) / kAnyWarps, 4096), batch * a.c.n_kv_heads, 2 * n_layers);
  launch_chained(k_rows_any<T, H, WRITE>, grid, dim3(kAnyWarps * 32), 0, s, a);
}

template <bool WRITE>
int move_rows(const dc_cache* c, const dc_cache_rows* r, void* stream) {
  int rc = op_check_cache(c);
  if (rc != DC_OK) return rc;
  if (!r || !r->k || !r->v) return op_fail(DC_ERR_INVALID_ARG, "null rows");
  if ((rc = op_check_dtype(c, r->dtype)) != DC_OK || (rc = op_check_batch(c, r->batch)) != DC_OK) return rc;
  if (r->layer < 0 || r->n_layers < 1 || r->layer > c->n_layers - r->n_layers)
    return op_fail(DC_ERR_SHAPE, "layers %d .. + %d of %d", r->layer, r->n_layers, c->n_layers);
  if ((rc = op_check_keys(c, r->batch, r->pos, r->n, c->max_ctx, "")) != DC_OK) return rc;
  if ((long long)r->batch * c->n_kv_heads > 65535 || r->n_layers > 32767) return op_fail(DC_ERR_UNSUPPORTED, "more than 65535 heads or 32767 layers in one call");
  RowsArgs a;
  a.c = *c; a.k = static_cast<char*>(r->k); a.v = static_cast<char*>(r->v); a.layer = r->layer;
  for (int i = 0; i < 5; ++i) { a.ks[i] = r->k_stride[i]; a.vs[i] = r->v_stride[i]; }
  int most = 0;
  for (int b = 0; b < DC_MAX_BATCH; ++b) {
    a.pos[b] = b < r->batch ? r->pos[b] : 0;
    a.n[b] = b < r->batch ? r->n[b] : 0;
    most = most > a.n[b] ? most : a.n[b];
  }
  if (most == 0) return DC_OK;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const bool f32 = r->dtype == DC_F32, q = c->dtype == DC_E4M3;
  if (f32 && q) launch<float, __nv_fp8_e4m3, WRITE>(a, r->batch, r->n_layers, most, s);
  else if (f32) launch<float, float, WRITE>(a, r->batch, r->n_layers, most, s);
  else if (q) launch<__nv_bfloat16, __nv_fp8_e4m3, WRITE>(a, r->batch, r->n_layers, most, s);
  else launch<__nv_bfloat16, __nv_bfloat16, WRITE>(a, r->batch, r->n_layers, most, s);
  return op_launched(WRITE ? "dc_cache_write" : "dc_cache_read");
}

}  // namespace
}  // namespace dc

extern "C" int dc_cache_write(const dc_cache* cache, const dc_cache_rows* rows, void* cuda_stream) {
  return dc::move_rows<true>(cache, rows, cuda_stream);
}
extern "C" int dc_cache_read(const dc_cache* cache, const dc_cache_rows* rows, void* cuda_stream) {
  return dc::move_rows<false>(cache, rows, cuda_stream);
}

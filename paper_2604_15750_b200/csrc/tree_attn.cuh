// Attention of drafted rows over a cache (dc_tree_attention): what its kernels share, and the CUDA-core one.
//
// The query rows of one kv head are its "lines": line m is row m / G, head m % G of the group of G = n_q_heads /
// n_kv_heads that reads it.  A unit of work is (sequence, kv head, a stretch of lines, a stretch of keys); stretches of keys are
// joined - by the CTAs of a cluster or, where they are too many for one, by k_tree_join - with the running maximum and sum that each of them leaves:
//     m = max_s m_s,   o = sum_s 2^(m_s - m) o_s / sum_s 2^(m_s - m) l_s
#pragma once
#include "ops.h"
#include "pdl.cuh"

namespace dc {

constexpr int kTreeTile = 128;   // keys: stretches are whole tiles

struct TreeArgs {
  dc_cache c;                    // k, v, scales moved to the layer
  const void* q;
  void* o;
  long long qs[3], os[3];        // sequence, row, head
  const uint32_t* mask;
  int words, max_rows;
  int nq, group, line_tiles;
  uint32_t group_inv;            // floor(2^32 / group) + 1: quotients of lines by the group without a division (tree_row)
  float scale_log2;              // scale * log2(e)
  int tiles;                     // of a stretch
  int joined;                    // stretches of the longest sequence; 1: none is written down
  int cluster;                   // they are the CTAs of a cluster, which joins them
  int base[DC_MAX_BATCH];        // lines (of all heads) before sequence b: where its partial results are
  int lines;                     // of all sequences
  int ctx[DC_MAX_BATCH], rows[DC_MAX_BATCH];
  float* part_o;                 // [stretch][line][head_dim]: sums not divided by l
  float2* part_ml;               // [stretch][line]: maximum (log2 units) and sum
  int32_t* status;
};

__device__ __forceinline__ int tree_stretches(const TreeArgs& a, int b) {
  const int t = (a.ctx[b] + a.rows[b] + kTreeTile - 1) / kTreeTile;
  return (t + a.tiles - 1) / a.tiles;
}
// row of line m: m / group, exactly where m * group < 2^32 (a sequence has 2^19 lines at most, a group 2^11)
__device__ __forceinline__ int tree_row(const TreeArgs& a, int m) { return a.group == 1 ? m : (int)__umulhi((uint32_t)m, a.group_inv); }
// place of (sequence, row, query head) among the lines
__device__ __forceinline__ int tree_line(const TreeArgs& a, int b, int r, int h) { return a.base[b] + r * a.nq + h; }

// ---- joins the stretches: a warp takes one (row, head) --------------------------------------------------
template <typename T>
__global__ void __launch_bounds__(256) k_tree_join(const __grid_constant__ TreeArgs a, const int batch) {
  pdl_wait();
  const int lane = threadIdx.x & 31, line = blockIdx.x * 8 + (threadIdx.x >> 5), hd = a.c.head_dim;
  if (line >= a.lines) return;
  int b = 0;
  while (b + 1 < batch && line >= a.base[b + 1]) ++b;
  const int n = tree_stretches(a, b);
  if (n <= 1) return;            // (its unit has written the output)
  const int r = (line - a.base[b]) / a.nq, h = (line - a.base[b]) % a.nq;
  // lane = stretch (32 at a time); a stretch without a key that the row sees has m = -infinity and sums of 0
  float top = -INFINITY;
  for (int s = lane; s < n; s += 32) top = fmaxf(top, a.part_ml[(size_t)s * a.lines + line].x);
#pragma unroll
  for (int i = 16; i >= 1; i >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, i));
  float o[8], l = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) o[i] = 0.f;
  for (int s0 = 0; s0 < n; s0 += 32) {
    float w = 0.f;
    if (s0 + lane < n) {
      const float2 ml = a.part_ml[(size_t)(s0 + lane) * a.lines + line];
      w = ml.x == -INFINITY ? 0.f : exp2f(ml.x - top);
      l = fmaf(w, ml.y, ml.x == -INFINITY ? l + ml.y : l);     // (NaN without a maximum: a NaN score, or a wait that ran out)
    }
    const int m = min(32, n - s0);
#pragma unroll 4
    for (int s = 0; s < m; ++s) {
      const float ws = __shfl_sync(0xffffffffu, w, s);
      const float* from = a.part_o + ((size_t)(s0 + s) * a.lines + line) * hd + lane;
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i * 32 + lane < hd) o[i] = fmaf(ws, from[i * 32], o[i]);
    }
  }
#pragma unroll
  for (int i = 16; i >= 1; i >>= 1) l += __shfl_xor_sync(0xffffffffu, l, i);
  T* dst = static_cast<T*>(a.o) + b * a.os[0] + r * a.os[1] + h * a.os[2];
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i * 32 + lane < hd) dst[i * 32 + lane] = op_to<T>(l == 0.f ? 0.f : o[i] / l);
}

// ---- CUDA cores: any head_dim and alignment, fp32 ----------------------------------------------------------
// grid (stretch, kv head, sequence * line tiles); 4 warps of 4 lines.  Scores: a lane takes a key; products with V: a lane
// takes dims.
constexpr int kTreeLines = 16, kTreeKeys = 32;
__host__ __device__ inline int tree_simt_smem(int hd) { return (kTreeLines * hd + kTreeKeys * (hd + 1) + hd * (kTreeKeys + 1)) * 4; }

template <typename T, typename H>
__global__ void __launch_bounds__(128) k_tree_simt(const __grid_constant__ TreeArgs a) {
  extern __shared__ float tree_smem[];
  const int b = blockIdx.z / a.line_tiles, R = a.rows[b], G = a.group, hd = a.c.head_dim, nkv = a.c.n_kv_heads;
  const int g = blockIdx.y, line0 = (blockIdx.z - b * a.line_tiles) * kTreeLines;
  const int keys = a.ctx[b] + R, k0 = blockIdx.x * a.tiles * kTreeTile, k1 = min(keys, k0 + a.tiles * kTreeTile);
  if (line0 >= R * G || k0 >= keys) return;
  float *qs = tree_smem, *ks = qs + kTreeLines * hd, *vs = ks + kTreeKeys * (hd + 1);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const size_t slot = (size_t)b * nkv + g;
  const H* K = static_cast<const H*>(a.c.k) + slot * a.c.max_ctx * hd;
  const H* V = static_cast<const H*>(a.c.v) + slot * a.c.max_ctx * hd;
  for (int i = threadIdx.x; i < kTreeLines * hd; i += 128) {
    const int m = line0 + i / hd;
    qs[i] = m < R * G ? op_f32(static_cast<const T*>(a.q)[b * a.qs[0] + (m / G) * a.qs[1] + (g * G + m % G) * a.qs[2] + i % hd]) : 0.f;
  }
  float top[4], l[4], o[4][8];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    top[j] = -INFINITY; l[j] = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) o[j][i] = 0.f;
  }
  for (int t = k0; t < k1; t += kTreeKeys) {
    __syncthreads();
    for (int i = threadIdx.x; i < kTreeKeys * hd; i += 128) {
      const int key = i / hd, d = i % hd;
      float x = 0.f;
      if (t + key < k1) {
        x = op_f32(K[(size_t)(t + key) * hd + d]);
        if (sizeof(H) == 1) x *= a.c.k_scale[slot * a.c.max_ctx + t + key];
      }
      ks[key * (hd + 1) + d] = x;
    }
    for (int i = threadIdx.x; i < kTreeKeys * hd; i += 128) {
      const int key = i % kTreeKeys, d = i / kTreeKeys;
      float x = 0.f;
      if (t + key < k1) {
        x = op_f32(V[(size_t)d * a.c.max_ctx + t + key]);
        if (sizeof(H) == 1) x *= a.c.v_scale[slot * a.c.max_ctx + t + key];
      }
      vs[d * (kTreeKeys + 1) + key] = x;
    }
    __syncthreads();
    float z[4] = {0.f, 0.f, 0.f, 0.f};
    const float* q = qs + warp * 4 * hd;
    for (int d = 0; d < hd; ++d) {
      const float x = ks[lane * (hd + 1) + d];
#pragma unroll
      for (int j = 0; j < 4; ++j) z[j] = fmaf(q[j * hd + d], x, z[j]);
    }
    const int key = t + lane, jd = key - a.ctx[b];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int m = line0 + warp * 4 + j;
      bool sees = key < k1 && m < R * G;
      if (sees && jd >= 0 && a.mask) sees = (a.mask[((size_t)b * a.max_rows + m / G) * a.words + (jd >> 5)] >> (jd & 31)) & 1u;
      z[j] = sees ? z[j] * a.scale_log2 : -INFINITY;
      float w = z[j];
#pragma unroll
      for (int i = 16; i >= 1; i >>= 1) w = fmaxf(w, __shfl_xor_sync(0xffffffffu, w, i));
      const float now = fmaxf(top[j], w);
      float p = 0.f;
      if (__any_sync(0xffffffffu, sees)) {     // (a NaN score makes the row NaN, whatever the maximum is)
        const float f = top[j] == -INFINITY ? 0.f : exp2f(top[j] - now);
        p = sees ? exp2f(z[j] - now) : 0.f;
        l[j] = l[j] * f + p;
#pragma unroll
        for (int i = 0; i < 8; ++i) o[j][i] *= f;
        top[j] = now;
      }
      z[j] = p;
    }
    for (int k = 0; k < kTreeKeys; ++k) {
      float p[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) p[j] = __shfl_sync(0xffffffffu, z[j], k);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int d = i * 32 + lane;
        if (d >= hd) break;
        const float x = vs[d * (kTreeKeys + 1) + k];
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (p[j] != 0.f) o[j][i] = fmaf(p[j], x, o[j][i]);     // (0 times what a key holds that the row does not see would be NaN)
      }
    }
  }
  const bool alone = tree_stretches(a, b) == 1;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int m = line0 + warp * 4 + j;
    float sum = l[j];
#pragma unroll
    for (int i = 16; i >= 1; i >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, i);
    if (m >= R * G) continue;
    const int r = m / G, h = g * G + m % G;
    if (alone) {
      T* dst = static_cast<T*>(a.o) + b * a.os[0] + r * a.os[1] + h * a.os[2];
      for (int i = 0; i < 8; ++i)
        if (i * 32 + lane < hd) dst[i * 32 + lane] = op_to<T>(sum == 0.f ? 0.f : o[j][i] / sum);
    } else {
      const size_t at = (size_t)blockIdx.x * a.lines + tree_line(a, b, r, h);
      if (lane == 0) a.part_ml[at] = make_float2(top[j], sum);
      for (int i = 0; i < 8; ++i)
        if (i * 32 + lane < hd) a.part_o[at * hd + i * 32 + lane] = o[j][i];
    }
  }
}

}  // namespace dc

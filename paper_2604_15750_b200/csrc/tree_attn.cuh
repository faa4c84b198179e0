// Attention of drafted rows over a cache (dc_tree_attention): what its kernels share, and the CUDA-core one.
//
// The query rows of one kv head are its "lines": line m is row m / G, head m % G of the group of G = n_q_heads /
// n_kv_heads that reads it.  A unit of work is (sequence, kv head, a stretch of lines, a stretch of keys); stretches of keys are
// joined - by the CTAs of a cluster or, where they are too many for one, by k_tree_join - with the running maximum and sum that each of them leaves:
//     m = max_s m_s,   o = sum_s 2^(m_s - m) o_s / sum_s 2^(m_s - m) l_s
#pragma once
#include "ops.h"
#include "pdl.cuh"
#include "tc_ptx.cuh"

namespace dc {

constexpr int kTreeTile = 128;   // keys: stretches are whole tiles
constexpr int kTreeMostKeys = 1 << 30;   // of a sequence: places of keys, and of the tiles behind the last one, are 32-bit numbers
constexpr int kTreeMostTiles = 1024;     // of a stretch over an 8-bit cache on the tensor cores (tc_tree.cuh)

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
  int stall;                     // DC_OPT_TEST_STALL_TREE
};

__device__ __forceinline__ int tree_stretches(const TreeArgs& a, int b) {
  const int t = (a.ctx[b] + a.rows[b] + kTreeTile - 1) / kTreeTile;
  return (t + a.tiles - 1) / a.tiles;
}
// row of line m: m / group, exactly where m * group < 2^32: a sequence has 2^19 lines at most
constexpr int kTreeMaxGroup = 2048;
__device__ __forceinline__ int tree_row(const TreeArgs& a, int m) { return a.group == 1 ? m : (int)__umulhi((uint32_t)m, a.group_inv); }
// place of (sequence, row, query head) among the lines
__device__ __forceinline__ int tree_line(const TreeArgs& a, int b, int r, int h) { return a.base[b] + r * a.nq + h; }

// ---- joins the stretches: a CTA takes one (row, head), its warps some of the stretches each ---------------------------
constexpr int kJoinWarps = 8;
template <typename T>
__global__ void __launch_bounds__(32 * kJoinWarps) k_tree_join(const __grid_constant__ TreeArgs a, const int batch) {
  __shared__ float part[kJoinWarps][256], sum[kJoinWarps];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, line = blockIdx.x, hd = a.c.head_dim;
  int b = 0;
  while (b + 1 < batch && line >= a.base[b + 1]) ++b;
  const int n = tree_stretches(a, b);
  pdl_wait();
  if (n <= 1) return;            // (its unit has written the output)
  // a stretch without a key that the row sees has m = -infinity and sums of 0
  float top = -INFINITY;
  for (int s = lane; s < n; s += 32) top = fmaxf(top, a.part_ml[(size_t)s * a.lines + line].x);
#pragma unroll
  for (int i = 16; i >= 1; i >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, i));
  float o[8], l = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) o[i] = 0.f;
#pragma unroll 4
  for (int s = warp; s < n; s += kJoinWarps) {
    const size_t at = (size_t)s * a.lines + line;
    const float2 ml = a.part_ml[at];
    const float w = ml.x == -INFINITY ? 0.f : exp2f(ml.x - top);
    l = ml.x == -INFINITY ? l + ml.y : fmaf(w, ml.y, l);     // (NaN without a maximum: a NaN score, or a wait that ran out)
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i * 32 + lane < hd) o[i] = fmaf(w, a.part_o[at * hd + i * 32 + lane], o[i]);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) part[warp][i * 32 + lane] = o[i];
  if (lane == 0) sum[warp] = l;
  __syncthreads();
  const int d = threadIdx.x, r = (line - a.base[b]) / a.nq, h = (line - a.base[b]) % a.nq;
  if (d >= hd) return;
  float x = 0.f;
  l = 0.f;
#pragma unroll
  for (int w = 0; w < kJoinWarps; ++w) { x += part[w][d]; l += sum[w]; }
  static_cast<T*>(a.o)[b * a.os[0] + r * a.os[1] + h * a.os[2] + d] = op_to<T>(l == 0.f ? 0.f : x / l);
}

// ---- CUDA cores, head_dim 64 or 128, cache on 16-byte boundaries ------------------------------------------
// grid (stretch, kv head, sequence * line tiles); 128 threads, 8 L lines (L of a thread: 8, or fewer where there are no more), 64 keys at
// a time.  In both products a thread has L lines x 4 keys or L lines x HD/16 dims in registers, two neighbours along the sum in one
// f32x2: with eight lines 12 16-byte loads from shared memory (an SM has four bytes a clock and lane) for 64 instructions of two multiply-adds.  Head_dim 64: the next keys' K
// and V are on their way (fp32: straight to shared memory) while these are worked on; 128, where two tiles have no room: the next K
// while V is worked on, and V while K is.  Drafted keys behind the last one that a line of the unit sees are left out.
// fp32, 64 rows of 4 heads a group, 4 x 2064 keys of 4 heads: head_dim 64 105 us, 128 183 us (2 lines x 4 keys a thread and single
// multiply-adds 137 and 264): 20.6 TFLOP/s, 28% of the multiply-adds' full rate, because two to three CTAs of four warps do not hide the
// latency of shared memory, and more have no room; bf16 the same (109 us), fp32 rows over e4m3, 128 dims 196 us (with 64 lines it spills).  9 rows, 14 x 2260 keys: 87 us (133).
constexpr int kSimtKeys = 64, kSimtThreads = 128;
__host__ __device__ constexpr int tree_simt_smem_hd(int hd, int l) {
  return (8 * l * (hd + 4) + (hd == 64 ? 2 : 1) * (kSimtKeys * (hd + 4) + hd * (kSimtKeys + 4)) + 8 * l * (kSimtKeys + 4)) * 4;
}
constexpr int tree_simt_ctas(int hd, int l) { return l == 1 ? 3 : l == 8 && hd == 128 ? 1 : 2; }     // of an SM, as shared memory has room
// 16 bytes of a cache as fp32
template <typename H> __device__ __forceinline__ void tree_wide(const uint4& w, float (&x)[16 / sizeof(H)]);
template <> __device__ __forceinline__ void tree_wide<__nv_bfloat16>(const uint4& w, float (&x)[8]) {
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(u[i] << 16); x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u); }
}
template <> __device__ __forceinline__ void tree_wide<__nv_fp8_e4m3>(const uint4& w, float (&x)[16]) {
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(u[i >> 1] >> (16 * (i & 1))), __NV_E4M3);
    const float2 f = __half22float2(__half2(h));
    x[2 * i] = f.x; x[2 * i + 1] = f.y;
  }
}
__device__ __forceinline__ void tree_copy16(float* to, const void* from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(ptx::smem_u32(to)), "l"(from) : "memory");
}
__device__ __forceinline__ void tree_copies_in() { asm volatile("cp.async.wait_all;" ::: "memory"); }

template <typename T, typename H, int HD, int L>
__global__ void __launch_bounds__(kSimtThreads, tree_simt_ctas(HD, L)) k_tree_simt_hd(const __grid_constant__ TreeArgs a) {
  constexpr bool F32 = sizeof(H) == 4;
  constexpr int kLines = 8 * L, kTiles = HD == 64 ? 2 : 1;        // tiles of K and V in shared memory
  constexpr int E = 16 / sizeof(H);                              // values of a load
  constexpr int NL = kSimtKeys * HD / E / kSimtThreads;          // loads a thread has of K, and of V
  constexpr int DPT = HD / 16, KP = HD + 4, VP = kSimtKeys + 4;  // dims a thread; row pitches in shared memory
  extern __shared__ float tree_smem[];
  __shared__ uint32_t poison[8];
  __shared__ int last_seen[kSimtThreads / 32];
  __shared__ uint32_t masks[kLines][8];      // of the unit's lines, bits of drafted keys
  const int b = blockIdx.z / a.line_tiles, R = a.rows[b], G = a.group, nkv = a.c.n_kv_heads;
  const int g = blockIdx.y, line0 = (blockIdx.z - b * a.line_tiles) * kLines, n = min(kLines, R * G - line0);
  const int ctx = a.ctx[b], keys = ctx + R, k0 = blockIdx.x * a.tiles * kTreeTile;
  int k1 = min(keys, k0 + a.tiles * kTreeTile);
  pdl_trigger();
  pdl_wait();
  if (n <= 0 || k0 >= keys) return;
  constexpr int kTileFloats = kSimtKeys * KP + HD * VP;
  float *qs = tree_smem, *ps = qs + kLines * KP, *tiles = ps + kLines * VP;
  auto k_at = [&](int t) { return tiles + (kTiles == 2 ? (t - k0) / kSimtKeys % 2 * kTileFloats : 0); };
  auto v_at = [&](int t) { return k_at(t) + kSimtKeys * KP; };
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;     // keys (dims) tx, tx + 16, .. of lines L ty .. + L - 1
  const size_t slot = (size_t)b * nkv + g;
  const H* K = static_cast<const H*>(a.c.k) + slot * a.c.max_ctx * HD;
  const H* V = static_cast<const H*>(a.c.v) + slot * a.c.max_ctx * HD;
  const float* k_scale = a.c.k_scale + slot * a.c.max_ctx;
  const float* v_scale = a.c.v_scale + slot * a.c.max_ctx;
  // (whole pieces of both: the cache goes on to a multiple of 64 keys)
  uint4 kw[F32 ? 1 : NL], vw[F32 ? 1 : NL];
  auto ask_k = [&](int t) {
    float* ks = k_at(t);
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int j = tid + kSimtThreads * i, key = j / (HD / E), d = j % (HD / E) * E;
      if constexpr (F32) tree_copy16(ks + key * KP + d, K + (size_t)(t + key) * HD + d);
      else kw[i] = *reinterpret_cast<const uint4*>(K + (size_t)(t + key) * HD + d);
    }
  };
  auto ask_v = [&](int t) {
    float* vs = v_at(t);
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int j = tid + kSimtThreads * i, d = j / (kSimtKeys / E), key = j % (kSimtKeys / E) * E;
      if constexpr (F32) tree_copy16(vs + d * VP + key, V + (size_t)d * a.c.max_ctx + t + key);
      else vw[i] = *reinterpret_cast<const uint4*>(V + (size_t)d * a.c.max_ctx + t + key);
    }
  };
  auto put_k = [&](int t) {
    if constexpr (!F32) {
      float* ks = k_at(t);
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        const int j = tid + kSimtThreads * i, key = j / (HD / E), d = j % (HD / E) * E;
        float x[E];
        tree_wide<H>(kw[i], x);
        const float sc = sizeof(H) == 1 ? k_scale[t + key] : 1.f;
#pragma unroll
        for (int e = 0; e < E; e += 4) *reinterpret_cast<float4*>(ks + key * KP + d + e) = make_float4(x[e] * sc, x[e + 1] * sc, x[e + 2] * sc, x[e + 3] * sc);
      }
    }
  };
  auto put_v = [&](int t) {
    if constexpr (!F32) {
      float* vs = v_at(t);
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        const int j = tid + kSimtThreads * i, d = j / (kSimtKeys / E), key = j % (kSimtKeys / E) * E;
        float x[E];
        tree_wide<H>(vw[i], x);
        if constexpr (sizeof(H) == 1) {
#pragma unroll
          for (int e = 0; e < E; ++e) x[e] *= v_scale[t + key + e];
        }
#pragma unroll
        for (int e = 0; e < E; e += 4) *reinterpret_cast<float4*>(vs + d * VP + key + e) = make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]);
      }
    }
  };
  ask_k(k0);
  if (!F32 || kTiles == 2) ask_v(k0);
  if (tid < 8) poison[tid] = 0;
  constexpr int kAsk = kLines * HD / kSimtThreads < 16 ? kLines * HD / kSimtThreads : 16;      // queries of a thread that are on their way at once
#pragma unroll 1
  for (int i0 = tid; i0 < kLines * HD; i0 += kAsk * kSimtThreads) {
    float x[kAsk];
#pragma unroll
    for (int i = 0; i < kAsk; ++i) {
      const int line = (i0 + i * kSimtThreads) / HD, d = i0 % HD, m = line0 + line, r = tree_row(a, m);
      x[i] = line < n ? op_f32(static_cast<const T*>(a.q)[b * a.qs[0] + r * a.qs[1] + (g * G + m - r * G) * a.qs[2] + d]) : 0.f;
    }
#pragma unroll
    for (int i = 0; i < kAsk; ++i) qs[(i0 + i * kSimtThreads) / HD * KP + i0 % HD] = x[i];
  }
  if (a.mask) {
    int last = -1;
    for (int i = tid; i < kLines * 8; i += kSimtThreads) {
      const int line = i >> 3, w = i & 7, left = R - 32 * w;
      uint32_t bits = 0u;
      if (line < n && left > 0) {
        bits = a.mask[((size_t)b * a.max_rows + tree_row(a, line0 + line)) * a.words + w];
        if (left < 32) bits &= (1u << left) - 1u;
      }
      masks[line][w] = bits;
      if (bits) last = max(last, 32 * w + 31 - __clz(bits));
    }
    last = __reduce_max_sync(0xffffffffu, last);
    if (tid % 32 == 0) last_seen[tid / 32] = last;
    __syncthreads();
    k1 = min(k1, ctx + max(max(last_seen[0], last_seen[1]), max(last_seen[2], last_seen[3])) + 1);
  }
  float top[L], sum[L];
  ptx::f32x2 o[L][DPT];
#pragma unroll
  for (int l = 0; l < L; ++l) {
    top[l] = -INFINITY; sum[l] = 0.f;
#pragma unroll
    for (int i = 0; i < DPT; ++i) o[l][i] = 0ull;
  }
  auto in_order = [&](int t) {
    if (t + kSimtKeys > k1 || (a.mask && t + kSimtKeys > ctx)) {
      // whatever the cache holds behind the last key, and a drafted key's values that are not finite: 0 times them would be NaN for
      // lines that do not see the key
      for (int i = tid; i < HD * kSimtKeys; i += kSimtThreads) {
        float& x = v_at(t)[i / kSimtKeys * VP + i % kSimtKeys];
        const int at = t + i % kSimtKeys;
        if (at >= k1) x = 0.f;
        else if (a.mask && at >= ctx && !(fabsf(x) <= 3.402823466e38f)) {
          x = 0.f;
          atomicOr(&poison[(at - ctx) >> 5], 1u << ((at - ctx) & 31));
        }
      }
      __syncthreads();
    }
  };
  const bool idle = tid / 32 * 2 * L >= n;      // (a warp without lines: the others have the pipes for themselves)
  for (int t = k0; t < k1; t += kSimtKeys) {
    const bool more = t + kSimtKeys < k1;
    const float *ks = k_at(t), *vs = v_at(t);
    put_k(t);
    if (kTiles == 2) put_v(t);
    tree_copies_in();
    __syncthreads();           // K (both) is there, and the keys before have been read
    if (kTiles == 2) {
      if (more) { ask_k(t + kSimtKeys); ask_v(t + kSimtKeys); }
      in_order(t);
    } else if (F32) {
      ask_v(t);
    } else {
      put_v(t);
      if (more) { ask_k(t + kSimtKeys); ask_v(t + kSimtKeys); }
    }
    if (!idle) {
      ptx::f32x2 z2[L][4];
#pragma unroll
      for (int l = 0; l < L; ++l)
#pragma unroll
        for (int e = 0; e < 4; ++e) z2[l][e] = 0ull;
#pragma unroll 4
      for (int d = 0; d < HD; d += 4) {
        ulonglong2 q[L], x[4];
#pragma unroll
        for (int l = 0; l < L; ++l) q[l] = *reinterpret_cast<const ulonglong2*>(qs + (L * ty + l) * KP + d);
        // (keys tx, tx + 16, ..: neighbours in shared memory rows go to different banks)
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = *reinterpret_cast<const ulonglong2*>(ks + (tx + 16 * e) * KP + d);
#pragma unroll
        for (int l = 0; l < L; ++l)
#pragma unroll
          for (int e = 0; e < 4; ++e) z2[l][e] = ptx::f2_fma(q[l].y, x[e].y, ptx::f2_fma(q[l].x, x[e].x, z2[l][e]));
      }
      // probabilities: the 16 threads of some lines have their keys
      const bool all = t + kSimtKeys <= min(ctx, k1) || (!a.mask && t + kSimtKeys <= k1);
#pragma unroll
      for (int l = 0; l < L; ++l) {
        float z[4], now = top[l];
        uint32_t sees = 0xfu;
        if (!all) {
          sees = 0u;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int key = t + tx + 16 * e, j = key - ctx;
            if (key < k1 && (j < 0 || !a.mask || (masks[L * ty + l][j >> 5] >> (j & 31) & 1u))) sees |= 1u << e;
          }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float odd;
          ptx::f2_unpack(z2[l][e], z[e], odd);
          z[e] = sees >> e & 1u ? (z[e] + odd) * a.scale_log2 : -INFINITY;
          now = fmaxf(now, z[e]);
        }
#pragma unroll
        for (int s = 8; s >= 1; s >>= 1) now = fmaxf(now, __shfl_xor_sync(0xffffffffu, now, s));
        const float f = top[l] == -INFINITY ? 0.f : exp2f(top[l] - now);
        sum[l] *= f;
        const ptx::f32x2 f2 = ptx::f2_pack(f, f);
#pragma unroll
        for (int i = 0; i < DPT; ++i) o[l][i] = ptx::f2_mul(o[l][i], f2);
        top[l] = now;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float p = sees >> e & 1u ? exp2f(z[e] - now) : 0.f;    // (a NaN score stays one)
          sum[l] += p;
          ps[(L * ty + l) * VP + tx + 16 * e] = p;
        }
      }
    }
    if (kTiles == 1) {
      tree_copies_in();
      __syncthreads();         // V is there, and K has been read
      if (F32 && more) ask_k(t + kSimtKeys);
      in_order(t);
    }
    if (idle) continue;
    __syncwarp();              // (a line's probabilities are made and read by the same half warp)
#pragma unroll 2
    for (int k = 0; k < kSimtKeys; k += 4) {
      ulonglong2 p[L];
#pragma unroll
      for (int l = 0; l < L; ++l) p[l] = *reinterpret_cast<const ulonglong2*>(ps + (L * ty + l) * VP + k);
#pragma unroll
      for (int i = 0; i < DPT; ++i) {
        const ulonglong2 x = *reinterpret_cast<const ulonglong2*>(vs + (tx + 16 * i) * VP + k);
#pragma unroll
        for (int l = 0; l < L; ++l) o[l][i] = ptx::f2_fma(p[l].y, x.y, ptx::f2_fma(p[l].x, x.x, o[l][i]));
      }
    }
    __syncwarp();
  }
  tree_copies_in();   // (of a unit that turned out to have no keys)
  __syncthreads();    // (what the last keys noted)
  const bool alone = tree_stretches(a, b) == 1;
#pragma unroll
  for (int l = 0; l < L; ++l) {
    float s = sum[l];
#pragma unroll
    for (int i = 8; i >= 1; i >>= 1) s += __shfl_xor_sync(0xffffffffu, s, i);
    if (L * ty + l >= n) continue;
    if (a.mask)
      for (int w = 0; w < a.words; ++w)
        if (masks[L * ty + l][w] & poison[w]) s = __uint_as_float(0x7fffffffu);
    const int m = line0 + L * ty + l, r = tree_row(a, m), h = g * G + m - r * G;
    const size_t at = (size_t)blockIdx.x * a.lines + tree_line(a, b, r, h);
    T* dst = static_cast<T*>(a.o) + b * a.os[0] + r * a.os[1] + h * a.os[2];
    if (!alone && tx == 0) a.part_ml[at] = make_float2(top[l], s);
#pragma unroll
    for (int i = 0; i < DPT; ++i) {
      float x, odd;
      ptx::f2_unpack(o[l][i], x, odd);
      x += odd;
      if (alone) dst[tx + 16 * i] = op_to<T>(s == 0.f ? 0.f : x / s);
      else a.part_o[at * HD + tx + 16 * i] = x;
    }
  }
}

// ---- CUDA cores: any head_dim and alignment, fp32 ----------------------------------------------------------
// The kernel for what the others do not take (64 rows of 4 heads a group, 4 x 2064 keys of 4 heads, fp32, head_dim 96: 940 us).
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
  pdl_trigger();
  pdl_wait();
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
        if (sees && p == 0.f) p = 1.4e-45f;    // (below all others, but V's infinities and NaN of a key that is seen arrive)
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

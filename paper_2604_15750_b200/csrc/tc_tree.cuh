// dc_tree_attention on tcgen05: bf16 rows, head_dim 128, a cache of bf16 or e4m3.  Keys on the 128 lanes, lines (tree_attn.cuh)
// on N columns, as in tc_attn_few.cuh:
//
//   S^T [128 keys x N lines]  = K Q^T
//   P^T                       = 2^(t - m),   t = scale * log2(e) * S     (0 where a line does not see the key)
//   O^T [128 dims x N lines] += V^T P^T      sums l += P^T over the keys beside it
//
// Few lines stream many keys: the cache's bytes are the bound (64 KB of bf16 or 32 KB of e4m3 a tile of 128 keys; at
// 6.5 TB/s an SM gets one in 2800 or 1400 clocks), and one thread per key does the softmax of N lines in less.
//
// An e4m3 cache goes to the tensor cores as it is (kind::f8f6f4), no byte of it is converted.  The other operand must have 8 bits
// too, and one such number has 3 or 4 significant bits, so it is given as a sum:
//   q = 2^e (hi + lo), e4m3 and e5m2, per line with the largest magnitude in [128, 256): hi leaves at most 8 units of a bf16 value's
//     last place, whole ones, which 3 bits hold, so down to 2^-13 of the largest every value is exact; what is below is off by
//     2^-14, 2^-21 of the largest, at most (lo as e4m3: 2^-9 and 2^-17); both products go to the same accumulator
//   P' = 2^(t + log2 v_scale + 11 - m) = three e5m2, whose exponents are those of fp16: the upper byte of the fp16 pattern, that of what
//     is left, and of what is left then the nearest: off by 2^-9 of the value, or 2^-17 where that is more, and the largest is
//     2^10 .. 2^15.8.  So keys count down to 2^-27 of a line's largest p v_scale, and 2^17 of them (a stretch has no more:
//     kTreeMostTiles) lose 2^-10 of it at most.  (Two e4m3 parts ended at 2^-17 of it while the sum still counted them: 16000
//     equal keys 2^-17 below one key lost a quarter of what they add.)
// The scales are factors of a key, and a thread has one key: K's goes into t, V's into P', so that the sum of a line
// takes P' / (2^11 v_scale).  The maximum m is that of t + log2 v_scale.
//
// m of a line is about the maximum of the first tile that it sees and moves only when a later tile has a t far above it
// (a vote of the four warps that hold a line's keys): then O and the sums are scaled by 2^(m_old - m_new).
//
// P lies in shared memory as the threads have it, a row of N values for a key (the product takes it with the lines as the
// contiguous axis): a thread stores 16 bytes at a time, where rows of keys would take a store for every value.
//
// Measured (device time of 21 passes): 16 x 4096 keys of 32 heads, 32 rows, e4m3, 566 MB: 102 us, 5.5 TB/s (119 us where passes go on for
// a second, 4.8); 8 x 900..1200 keys, 24 rows, 77 MB: 21.2 us (3.6 TB/s; a unit's start and end are a third); 4 x 768 keys of 4 heads,
// 64 rows of 7 heads a group, bf16: 11.0 us (seven tiles one after the other, 1250 clk each); one row over 512 keys of 32 heads:
// 8.3 us.  The third part of P costs 1 to 5% of these over e4m3.
//
// Why N = 32, 64 or 128: a column costs softmax time whether it has a line or not, and every further unit streams the keys again.
// 32 lines and e4m3 leave room for two CTAs on an SM, whose starts and softmax overlap.  128 lines take in 64 KB of bf16 a tile for
// four times as many as 32: 4 x 4000 keys, 128 rows of 7 heads 49 us, with 64 lines 67.  Over e4m3 the
// softmax bounds: a tile of 64 lines takes 0.80 us of 128, 1.01 alone, 1.25 as two of 32 (12 x 4635 keys of 8 heads, 121 rows of 4 heads a
// group 225 us).  Which one is taken: kCost8, kCost16 (tree_attn.cu).
//
// Warps: 0 = TMA producer (K and V^T rings), 1 = TMEM owner and issuer of S^T, 2 = issuer of O^T, which first puts V^T tiles in order
// (clears keys beyond the last; a drafted key's values that are not finite are cleared and noted, because 0 times them
// would be NaN for lines that do not see the key), 3 = factors that the scales of e4m3 keys make, 4 .. = softmax and output, four
// warps for every 16 lines, or 32 of 128 (a warp reads the quarter of TMEM's lanes that its number says).
#pragma once
#include "tc_attn_parts.cuh"
#include "tree_attn.cuh"

namespace dc {

template <int N, bool Q8>
struct TreeTc {
  static constexpr int kLines = N == 128 ? 32 : 16;             // lines of a softmax warp, in chunks of 16
  static constexpr int kGroups = N / kLines, kThreads = 128 + 128 * kGroups;
  static constexpr int kSlot = Q8 ? kSub : 2 * kSub;           // a tile of K or of V^T
  // slots of the rings, as shared memory has room (128 lines over e4m3: 2 + 3 or 3 + 2, the same to 0.5%)
  static constexpr int kRingK = N == 32 ? (Q8 ? 2 : 3) : N == 64 ? (Q8 ? 4 : 3) : 2;
  static constexpr int kP = Q8 && N >= 64 ? 2 : 1;             // tiles of P: with two no warp waits for the product before
  static constexpr int kRingV = N == 32 || (Q8 && N == 128) ? 3 : kRingK;
  // Half of the softmax warps turn scores into P while the other half reads and scales its scores: left alone all warps do the
  // same at the same time, and the unit for 2^x is idle for the rest (with two parts of P a tile of 128 x 128 1.80 -> 1.46 us, 64
  // lines 1.07 -> 0.97; with 128 lines over bf16 1.25 -> 1.68)
  static constexpr bool kTurns = Q8 && N >= 64;
  static constexpr int kResident = Q8 && N == 32 ? 2 : 1;      // CTAs of an SM
  static constexpr int kOperand = N * 256;                     // bytes of Q
  static constexpr int kPTile = (Q8 ? 3 : 2) * N * 128;        // bytes of P: three parts, or bf16
  static constexpr int kCtl = ((N == 128 ? 5 : 3) + (Q8 ? 4 : 0)) * 1024;
  static constexpr int kSmem = kOperand + kP * kPTile + (kRingK + kRingV) * kSlot + kCtl;
  // P: the rows of the keys, of 128 bytes at most; a second half of the lines lies behind (bf16, 128 lines)
  static constexpr int kPRow = Q8 ? N : N == 128 ? 128 : 2 * N;
  static constexpr int kColO = 2 * N, kCols = N == 32 ? 128 : N == 64 ? 256 : 512;   // TMEM: S^T twice, O^T
  static_assert(kColO + N <= kCols && kSmem <= 232448 && kResident * (kSmem + 1024) <= 233472, "TMEM, shared memory");
  static_assert(N * 512 <= kOperand + kP * kPTile, "the output of a stretch in fp32 lies where Q and P were");
};
// P' over e4m3 is 2^15.8 at most (e5m2 ends at 1.75 x 2^15): m is set 1 above the maximum, where P' is 2^11, which leaves 5.8 for later
// tiles, and each time that m moves costs about half a tile.
constexpr float kHeadBf16 = 40.f, kHeadE4m3 = 15.8f, kAhead = 1.f, kUp = 11.f;

template <int N, bool Q8>
struct TreeCtl {
  uint64_t k_full[4], k_empty[4], v_full[4], v_empty[4], s_full[2], s_empty[2], p_full[2], p_empty[2], turn[2];   // turn: a half is done with 2^x
  uint64_t ended[2];                     // given up: the issuers' products
  uint32_t tmem_base;
  int abort_flag, late_flag, poisoned;
  uint32_t poison[8];                    // drafted keys whose V is not finite
  alignas(16) float nm[N];               // the lines' maxima, negative (log2 units)
  alignas(16) float fac[N];              // what the sums are scaled by when they move; at the end 1 / l
  long long at[N];                       // places of the lines in o or part_o
  alignas(16) float rs[N];               // e4m3: 2^e of a line's q
  alignas(16) float part[4][N];
  float4 key[2][Q8 ? kTreeTile : 1];     // e4m3: factor of a key's scores, log2 of V's scale, factor of the sums
};

// Sum of v[col] over the lanes of a warp, 16 columns at once: lane i returns that of column i % 16.
__device__ __forceinline__ float tree_sum(float (&v)[16], int lane) {
#pragma unroll
  for (int i = 0; i < 16; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], 16);
#pragma unroll
  for (int s = 8; s >= 1; s >>= 1) {
    const bool upper = (lane & s) != 0;
#pragma unroll
    for (int i = 0; i < s; ++i) {
      const float send = upper ? v[i] : v[i + s], keep = upper ? v[i + s] : v[i];
      v[i] = keep + __shfl_xor_sync(0xffffffffu, send, s);
    }
  }
  return v[0];
}
// 32 lanes x 4 consecutive columns of TMEM
__device__ __forceinline__ void tree_tmem_ld4(uint32_t at, float (&v)[4]) {
  uint32_t* r = reinterpret_cast<uint32_t*>(v);
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void tree_tmem_st4(uint32_t at, float x, float y, float z, float w) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1, %2, %3, %4};"
               ::"r"(at), "r"(__float_as_uint(x)), "r"(__float_as_uint(y)), "r"(__float_as_uint(z)), "r"(__float_as_uint(w)) : "memory");
}
// the same place in the shared memory of another CTA of the cluster
__device__ __forceinline__ float tree_remote(const float* p, int rank) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(ptx::mapa_shared(ptx::smem_u32(p), (uint32_t)rank)) : "memory");
  return v;
}
__device__ __forceinline__ float4 tree_remote4(const void* p, int rank) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
               : "r"(ptx::mapa_shared(ptx::smem_u32(p), (uint32_t)rank)) : "memory");
  return v;
}
// largest value of a warp, NaN passed over
__device__ __forceinline__ float tree_max(float x) {
  float r;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));
  return r;
}

// D (+)= A B: bf16 operands 16 deep, or e4m3 32 deep (split descriptors, as umma_bf16_lo; A and B with upper halves of their own)
template <bool Q8>
__device__ __forceinline__ void tree_umma(uint32_t d, uint32_t a_lo, uint32_t a_hi, uint32_t b_lo, uint32_t b_hi, uint32_t idesc, uint32_t accumulate) {
  if (Q8)
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\t"
        "mov.b64 da, {%1, %2};\n\tmov.b64 db, {%3, %4};\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], da, db, %5, p;\n\t}"
        ::"r"(d), "r"(a_lo), "r"(a_hi), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accumulate) : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\t"
        "mov.b64 da, {%1, %2};\n\tmov.b64 db, {%3, %4};\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %5, p;\n\t}"
        ::"r"(d), "r"(a_lo), "r"(a_hi), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accumulate) : "memory");
}
// 128 x n, fp32 sums; B with its rows (N) or with its columns (the depth) as the contiguous axis; over e4m3 B is e4m3 or e5m2
template <bool Q8>
__device__ __forceinline__ uint32_t tree_idesc(int n, bool rows_contiguous, bool e5m2) {
  return (1u << 4) | (Q8 ? (e5m2 ? 1u << 10 : 0u) : (1u << 7) | (1u << 10)) | (rows_contiguous ? 1u << 16 : 0u) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
}
// Upper half of the descriptor of P: rows (keys) of `row` bytes = one swizzle span, 8 of them a group
__device__ __forceinline__ uint32_t tree_p_desc_hi(int row) {
  return (uint32_t)(8 * row >> 4) | (1u << 14) | ((row == 128 ? 2u : row == 64 ? 4u : 6u) << 29);
}

__device__ __forceinline__ uint32_t tree_fp8x2(float x0, float x1, __nv_fp8_interpretation_t as) {
  return __nv_cvt_float2_to_fp8x2(make_float2(x0, x1), __NV_SATFINITE, as);
}
// Four values >= 0, two in an f16x2, as sums of three e5m2: an e5m2 is the upper byte of an fp16.  (A NaN stays one in the first part.)
__device__ __forceinline__ __half2 tree_upper(__half2 x) {
  const uint32_t w = *reinterpret_cast<const uint32_t*>(&x) & 0xff00ff00u;
  return *reinterpret_cast<const __half2*>(&w);
}
__device__ __forceinline__ uint32_t tree_bytes(__half2 x, __half2 y, uint32_t add) {    // (fp16 patterns are below 2^15: no carry)
  return __byte_perm(*reinterpret_cast<const uint32_t*>(&x) + add, *reinterpret_cast<const uint32_t*>(&y) + add, 0x7531);
}
__device__ __forceinline__ void tree_split4(__half2 x, __half2 y, uint32_t (&part)[3]) {
  part[0] = tree_bytes(x, y, 0u);
  x = __hsub2(x, tree_upper(x)); y = __hsub2(y, tree_upper(y));
  part[1] = tree_bytes(x, y, 0u);
  x = __hsub2(x, tree_upper(x)); y = __hsub2(y, tree_upper(y));
  part[2] = tree_bytes(x, y, 0x00800080u);       // (half of what the lower byte can hold: to the nearest)
}
__device__ __forceinline__ __half2 tree_half2(uint32_t e4m3x2) {
  return __half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)e4m3x2, __NV_E4M3));
}

// A bounded wait as ptx::mbar_wait, without the hint that lets a try sleep: the warps here wait little, and a try with the
// hint is a loop of its own, whose instructions the softmax warps of the other CTA on the SM would have to share with.
__device__ __forceinline__ bool tree_try(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred P;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 P, [%1], %2;\n\t"
      "selp.b32 %0, 1, 0, P;\n\t}"
      : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  return ok != 0;
}
__device__ __noinline__ bool tree_wait_on(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
  const unsigned long long t0 = ptx::globaltimer();
  uint32_t polls = 0;
  while (!tree_try(bar, parity)) {
    if ((++polls & 0xff) == 0) {
      if (*abort_flag) return false;
      if (ptx::globaltimer() - t0 > ptx::g_wait_limit_ns) {
        *abort_flag = 1;
        return false;
      }
    }
  }
  return true;
}
__device__ __forceinline__ bool tree_wait(uint64_t* bar, uint32_t parity, volatile int* abort_flag) {
  const uint32_t at = ptx::smem_u32(bar);
  return tree_try(at, parity) || tree_wait_on(at, parity, abort_flag);
}
// The same for a whole warp, whose lanes agree: the vote keeps the branch of the usual case uniform.
__device__ __forceinline__ bool tree_wait_warp(uint64_t* bar, uint32_t parity, volatile int* abort_flag) {
  const uint32_t at = ptx::smem_u32(bar);
  return __all_sync(0xffffffffu, tree_try(at, parity)) || __all_sync(0xffffffffu, tree_wait_on(at, parity, abort_flag));
}
__device__ __forceinline__ float tree_rcp(float x) {
  float y;
  asm("rcp.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float tree_lg2(float x) {
  float y;
  asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Queries of a CTA's lines, items of 8 dims of a line: the loads, and what becomes of them in shared memory (rows of
// 128 bytes with the 128-byte swizzle; e4m3: hi, then lo).
template <int N, bool Q8>
__device__ __forceinline__ void tree_load_q(const TreeArgs& a, int b, int g, int line0, int n, int vec, int item, uint4& w) {
  const int line = item >> 4, c = item & 15;
  w = make_uint4(0u, 0u, 0u, 0u);
  if (line >= n) return;
  const int m = line0 + line, r = tree_row(a, m), h = g * a.group + m - r * a.group;
  const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(a.q) + b * a.qs[0] + r * a.qs[1] + h * a.qs[2] + c * 8;
  if (vec) {
    w = *reinterpret_cast<const uint4*>(q);
  } else {
    auto two = [&](int e) { return (uint32_t)__bfloat16_as_ushort(q[e]) | (uint32_t)__bfloat16_as_ushort(q[e + 1]) << 16; };
    w = make_uint4(two(0), two(2), two(4), two(6));
  }
}
template <int N, bool Q8>
__device__ __forceinline__ void tree_store_q(int item, const uint4& v, uint8_t* Qs, float* rs) {    // (whole warps)
  const int line = item >> 4, c = item & 15;
  if (!Q8) {
    *reinterpret_cast<uint4*>(Qs + (c >> 3) * (N * 128) + line * 128 + (((c & 7) ^ (line & 7)) << 4)) = v;
    return;
  }
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  uint32_t top = 0;     // magnitudes order as their patterns do
#pragma unroll
  for (int e = 0; e < 4; ++e) top = max(top, max(w[e] & 0x7fffu, (w[e] >> 16) & 0x7fffu));
#pragma unroll
  for (int s = 8; s >= 1; s >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, s));
  const int ex = max((int)(top >> 7), 20) - 127;            // of the largest magnitude
  const float f = __uint_as_float((uint32_t)(127 + 7 - ex) << 23);
  if (c == 0) rs[line] = top >= 0x7f80u ? __uint_as_float(0x7fffffffu) : __uint_as_float((uint32_t)(127 - 7 + ex) << 23);
  uint32_t hi[2] = {0u, 0u}, lo[2] = {0u, 0u};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float x0 = __uint_as_float(w[e] << 16) * f, x1 = __uint_as_float(w[e] & 0xffff0000u) * f;
    const uint32_t h = tree_fp8x2(x0, x1, __NV_E4M3);
    const float2 r = __half22float2(tree_half2(h));
    hi[e >> 1] |= h << (16 * (e & 1));
    lo[e >> 1] |= tree_fp8x2(x0 - r.x, x1 - r.y, __NV_E5M2) << (16 * (e & 1));
  }
  uint8_t* at = Qs + line * 128 + (((c >> 1) ^ (line & 7)) << 4) + (c & 1) * 8;
  *reinterpret_cast<uint2*>(at) = make_uint2(hi[0], hi[1]);
  *reinterpret_cast<uint2*>(at + N * 128) = make_uint2(lo[0], lo[1]);
}

// Address of the 16-byte piece of row rr of a V^T tile: pieces of 16 (e4m3) or 8 keys
template <bool Q8>
__device__ __forceinline__ uint4* tree_v_piece(uint8_t* tile, int rr, int piece) {
  if (Q8) return reinterpret_cast<uint4*>(tile + rr * 128 + ((piece ^ (rr & 7)) << 4));
  return reinterpret_cast<uint4*>(tile + (piece >> 3) * kSub + rr * 128 + (((piece & 7) ^ (rr & 7)) << 4));
}

// Values of drafted keys (in the tile: from .. to - 1) that are not finite: cleared, and their keys noted.  Looked for first, four
// rows a lane at a time, because they are hardly ever there and the last product waits for this.
template <bool Q8>
__device__ __forceinline__ uint32_t tree_not_finite(uint32_t w) {    // top bit of each such value
  return Q8 ? ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u : ((w & 0x7fff7fffu) + 0x00800080u) & 0x80008000u;
}
template <bool Q8>
__device__ __noinline__ void tree_clear_not_finite(uint8_t* tile, int from, int to, int first_draft, uint32_t* poison) {
  constexpr int KPP = Q8 ? 16 : 8, KPW = Q8 ? 4 : 2;     // keys of a piece, of a word
  for (int pc = from / KPP; pc * KPP < to; ++pc)
    for (int rr = threadIdx.x & 31; rr < 128; rr += 32) {
      uint32_t* at = reinterpret_cast<uint32_t*>(tree_v_piece<Q8>(tile, rr, pc));
#pragma unroll 1
      for (int i = 0; i < 4; ++i) {
        uint32_t w = at[i];
        const uint32_t bad = tree_not_finite<Q8>(w);
        for (int e = 0; e < KPW && bad; ++e) {
          const int key = pc * KPP + i * KPW + e, j = key - from + first_draft;
          const uint32_t bits = (Q8 ? 0xffu : 0xffffu) << (e * (32 / KPW));
          if ((bad & bits) && key >= from && key < to) {
            w &= ~bits;
            atomicOr(&poison[j >> 5], 1u << (j & 31));
          }
        }
        at[i] = w;
      }
    }
}
template <bool Q8>
__device__ __forceinline__ void tree_clean_v(uint8_t* tile, int from, int to, int first_draft, uint32_t* poison, int* poisoned) {
  constexpr int KPP = Q8 ? 16 : 8;
  const int lane = threadIdx.x & 31;
  uint32_t any = 0;
#pragma unroll 1
  for (int pc = from / KPP; pc * KPP < to; ++pc) {
    uint4 w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = *tree_v_piece<Q8>(tile, lane + 32 * i, pc);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      any |= tree_not_finite<Q8>(w[i].x) | tree_not_finite<Q8>(w[i].y) | tree_not_finite<Q8>(w[i].z) | tree_not_finite<Q8>(w[i].w);
  }
  if (__any_sync(0xffffffffu, any != 0)) {     // (it may be of a key of the context, seen by all)
    tree_clear_not_finite<Q8>(tile, from, to, first_draft, poison);
    if (lane == 0) *poisoned = 1;
  }
}

// Clears keys valid .. up to what the product takes (its steps are 32 keys of e4m3) in row rr
__device__ __forceinline__ void tree_clear_v8(uint8_t* tile, int rr, int valid) {
  const int c = valid >> 4, k = valid & 15;
  uint4* at = tree_v_piece<true>(tile, rr, c);
  uint4 w = *at;
  auto kept = [&](int first) { const int n = k - first; return n >= 4 ? 0xffffffffu : n <= 0 ? 0u : (1u << (8 * n)) - 1u; };
  w.x &= kept(0); w.y &= kept(4); w.z &= kept(8); w.w &= kept(12);
  *at = w;
  if ((c & 1) == 0) *tree_v_piece<true>(tile, rr, c + 1) = make_uint4(0, 0, 0, 0);
}

template <int N, bool Q8>
__global__ void __launch_bounds__(TreeTc<N, Q8>::kThreads, TreeTc<N, Q8>::kResident)
k_tree_tc(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const __grid_constant__ TreeArgs a, const int vec_q, const int vec_o) {
  using C = TreeTc<N, Q8>;
  extern __shared__ uint8_t smem_tree[];
  const int g = blockIdx.y, G = a.group, nkv = a.c.n_kv_heads;
  const int b = a.line_tiles == 1 ? (int)blockIdx.z : (int)blockIdx.z / a.line_tiles, line0 = ((int)blockIdx.z - b * a.line_tiles) * N;
  const int R = a.rows[b], n = min(N, R * G - line0);
  const int ctx = a.ctx[b], keys = ctx + R, tile0 = blockIdx.x * a.tiles;
  const int T = min((keys + kTreeTile - 1) / kTreeTile - tile0, a.tiles);
  // (a cluster's barriers wait for the CTAs that are still there, and nobody reads the shared memory of one without keys)
  if (n <= 0 || T <= 0) { pdl_wait(); return; }
  uint8_t *Qs = smem_tree, *Ps = Qs + C::kOperand, *kring = Ps + C::kP * C::kPTile, *vring = kring + C::kRingK * C::kSlot;
  TreeCtl<N, Q8>& c = *reinterpret_cast<TreeCtl<N, Q8>*>(vring + C::kRingV * C::kSlot);
  static_assert(sizeof(TreeCtl<N, Q8>) <= C::kCtl, "control block");
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 96) { ptx::prefetch_tmap(&map_k); ptx::prefetch_tmap(&map_v); }
  if ((ptx::smem_u32(smem_tree) & 1023u) != 0) {   // (it is all the shared memory there is and starts on such a boundary)
    pdl_wait();
    if (threadIdx.x == 0 && a.status) atomicExch(a.status, DC_ERR_UNSUPPORTED);
    return;
  }
  if (threadIdx.x == 0) {
    c.abort_flag = 0; c.late_flag = 0; c.poisoned = 0;
    for (int i = 0; i < C::kRingK; ++i) { ptx::mbar_init(&c.k_full[i], 1); ptx::mbar_init(&c.k_empty[i], 1); }
    for (int i = 0; i < C::kRingV; ++i) { ptx::mbar_init(&c.v_full[i], 1); ptx::mbar_init(&c.v_empty[i], 1); }
    for (int i = 0; i < 2; ++i) { ptx::mbar_init(&c.s_full[i], Q8 ? 2 : 1); ptx::mbar_init(&c.s_empty[i], 4 * C::kGroups); }
    for (int i = 0; i < C::kP; ++i) { ptx::mbar_init(&c.p_full[i], 4 * C::kGroups); ptx::mbar_init(&c.p_empty[i], 1); }   // (full: the softmax warps)
    for (int i = 0; i < 2; ++i) { ptx::mbar_init(&c.turn[i], 2 * C::kGroups); ptx::mbar_init(&c.ended[i], 1); }
    ptx::fence_barrier_init();
    ptx::fence_proxy_async_smem();
  }
  pdl_wait();      // (pdl.cuh: nothing of the caller's memory is read or written before)

  // the queries are asked for before the tiles of all CTAs fill the way from memory (by warps 1 ..: warp 0 asks for the tiles)
  constexpr int kAskers = C::kThreads - 32, kItems = (N * 16 + kAskers - 1) / kAskers;
  uint4 q[kItems];
#pragma unroll
  for (int i = 0; i < kItems; ++i) {
    const int item = (int)threadIdx.x - 32 + i * kAskers;
    if (warp > 0 && item < N * 16) tree_load_q<N, Q8>(a, b, g, line0, n, vec_q, item, q[i]);
  }
  // softmax warps: who sees this thread's key, a bit for each of the warp's lines: tiles without drafted keys by the keys' number
  // alone, the (at most three) others by the mask
  const int draft0 = ctx / kTreeTile;
  uint32_t seen[3], of_line[3];
  float ks[4], vs[4];     // warp 3: the scales of keys lane, lane + 32, .. of a tile
  const size_t scales = (size_t)(b * nkv + g) * a.c.max_ctx + (size_t)tile0 * kTreeTile + lane;
  auto load_scales = [&](int j) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bool there = (tile0 + j) * kTreeTile + 32 * i + lane < keys;
      ks[i] = there ? a.c.k_scale[scales + (size_t)j * kTreeTile + 32 * i] : 0.f;
      vs[i] = there ? a.c.v_scale[scales + (size_t)j * kTreeTile + 32 * i] : 1.f;
    }
  };
  if (Q8 && warp == 3) load_scales(0);
  if (warp >= 4) {
    const int quarter = warp & 3, col0 = ((warp - 4) >> 2) * C::kLines, line = line0 + col0 + lane % C::kLines;
    const uint32_t* row = a.mask && line < line0 + n ? a.mask + ((size_t)b * a.max_rows + tree_row(a, line)) * a.words : nullptr;
#pragma unroll
    for (int i = 0; i < 3; ++i) {      // lane = line: the 32 keys of the warp's quarter
      const int jd = (draft0 + i) * kTreeTile + quarter * 32 - ctx, w = jd >> 5;
      const bool here = draft0 + i >= tile0 && draft0 + i < tile0 + T;
      auto word = [&](int x) { return row && here && x >= 0 && x < a.words ? row[x] : 0xffffffffu; };
      of_line[i] = __funnelshift_r(word(w), word(w + 1), jd & 31);
      if (R - jd < 32) of_line[i] &= R - jd > 0 ? (1u << (R - jd)) - 1u : 0u;
    }
  }
  // a tile of K or of V^T into its slot (one thread)
  const int krow = (b * nkv + g) * a.c.max_ctx, vrow = (b * nkv + g) * kHd;
  auto load_k = [&](int j) {
    const int s = j % C::kRingK, key = (tile0 + j) * kTreeTile;
    uint8_t* dst = kring + (size_t)s * C::kSlot;
    ptx::mbar_expect_tx(&c.k_full[s], C::kSlot);
    ptx::tma_load_2d(dst, &map_k, &c.k_full[s], 0, krow + key);
    if (!Q8) ptx::tma_load_2d(dst + kSub, &map_k, &c.k_full[s], 64, krow + key);
  };
  auto load_v = [&](int j) {
    const int s = j % C::kRingV, key = (tile0 + j) * kTreeTile;
    uint8_t* dst = vring + (size_t)s * C::kSlot;
    ptx::mbar_expect_tx(&c.v_full[s], C::kSlot);
    ptx::tma_load_2d(dst, &map_v, &c.v_full[s], key, vrow);
    if (!Q8) ptx::tma_load_2d(dst + kSub, &map_v, &c.v_full[s], key + 64, vrow);
  };
  const bool silent = a.stall == 1 || (a.stall == 3 && blockIdx.x == 1);     // (test hook: this CTA asks for no tile)
  if (threadIdx.x == 0 && !silent) {
    // the first tiles are on their way while the CTA sets up, and only these: the others would be in the way of the queries of the
    // CTAs that start later (8 x 1200 keys, 24 rows: the whole rings 22.6 us, one K tile 21.4, one of each 21.2)
    load_k(0);
    load_v(0);
  }
  if (threadIdx.x < 8) c.poison[threadIdx.x] = 0u;
  static_assert(N <= 128, "a thread a line");
  if (threadIdx.x < N) c.nm[threadIdx.x] = (int)threadIdx.x < n ? INFINITY : -INFINITY;   // (columns without a line: P = 0)
  if (warp == 1) {
    __syncwarp();
    ptx::tmem_alloc(&c.tmem_base, C::kCols);
    ptx::tmem_relinquish();
  }
#pragma unroll
  for (int i = 0; i < kItems; ++i) {       // (N * 16 is a multiple of 32: whole warps)
    const int item = (int)threadIdx.x - 32 + i * kAskers;
    if (warp > 0 && item < N * 16) tree_store_q<N, Q8>(item, q[i], Qs, c.rs);
  }
  if (warp >= 4) {
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      seen[i] = C::kLines == 16 ? 0xffff0000u : 0u;
      if (draft0 + i >= tile0 && draft0 + i < tile0 + T) {
#pragma unroll
        for (int e = 0; e < C::kLines; ++e) seen[i] |= ((__shfl_sync(0xffffffffu, of_line[i], e) >> lane) & 1u) << e;
      }
    }
  }
  ptx::fence_proxy_async_smem();
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t tmem_base = c.tmem_base;
  pdl_trigger();   // (the join; not before the allocation: pdl.cuh)

  int* abort_flag = &c.abort_flag;
  int loads_k = 0, loads_v = 0;   // of the producer thread
  auto valid_keys = [&](int j) { return min(kTreeTile, keys - (tile0 + j) * kTreeTile); };
  // V^T tiles that are put in order before their product: the stretch's last ones
  auto drafted = [&](int j) { return a.mask && (tile0 + j) * kTreeTile + valid_keys(j) > ctx; };
  auto ragged = [&](int j) { return (valid_keys(j) & (Q8 ? 31 : 15)) != 0; };
  if (warp == 0) {
    if (lane == 0) {
      // ---------------- TMA producer ----------------
      loads_k = loads_v = silent ? 0 : 1;
      while (!silent && a.stall != 2 && (loads_k < T || loads_v < T)) {
        if (loads_k < T) {
          if (loads_k >= C::kRingK && !tree_wait(&c.k_empty[loads_k % C::kRingK], ((uint32_t)(loads_k / C::kRingK) & 1u) ^ 1u, abort_flag)) break;
          load_k(loads_k++);
        }
        if (loads_v < T) {
          if (loads_v >= C::kRingV && !tree_wait(&c.v_empty[loads_v % C::kRingV], ((uint32_t)(loads_v / C::kRingV) & 1u) ^ 1u, abort_flag)) break;
          load_v(loads_v++);
        }
      }
    }
  } else if (warp == 1 || warp == 2) {
    // ---------------- issuers of S^T = K Q^T (warp 1) and O^T (+)= V^T P^T (warp 2) ----------------
    const bool pv = warp == 2;
    const uint32_t idesc = tree_idesc<Q8>(N, pv, pv), idesc_lo = tree_idesc<Q8>(N, pv, true), a_hi = ptx::smem_desc_hi32(), b_hi = pv ? tree_p_desc_hi(C::kPRow) : a_hi;
    // (two halves of lines lie 128 rows of 128 bytes apart)
    const uint32_t b_lo = pv && !Q8 && N == 128 ? (1024u << 16) | ((ptx::smem_u32(Ps) >> 4) & 0x3fffu) : ptx::smem_desc_lo(ptx::smem_u32(pv ? Ps : Qs));
    const uint32_t ring_lo = ptx::smem_desc_lo(ptx::smem_u32(pv ? vring : kring));
    // from one product to the next: Q goes on in its row, P by the rows of 16 (32) keys; the parts lie behind one another
    const uint32_t b_step = pv ? (uint32_t)((Q8 ? 32 : 16) * C::kPRow >> 4) : 2u, b_half = pv ? 4u * b_step : (uint32_t)(N * 128 >> 4);
    bool ok = true;
    for (int j = 0; j < T && ok; ++j) {
      const int s = pv ? j % C::kRingV : j % C::kRingK;
      if (pv) {
        ok = tree_wait_warp(&c.v_full[s], (uint32_t)(j / C::kRingV) & 1u, abort_flag);
        if (!ok) break;
        if (drafted(j) || ragged(j)) {     // (while the softmax warps make P)
          const int key0 = (tile0 + j) * kTreeTile, valid = valid_keys(j);
          uint8_t* tile = vring + (size_t)s * C::kSlot;
          if (ragged(j))
            for (int rr = lane; rr < 128; rr += 32) {
              if (Q8) tree_clear_v8(tile, rr, valid);
              else attn_clear_v(tile, rr, valid);
            }
          if (drafted(j)) tree_clean_v<Q8>(tile, max(0, ctx - key0), valid, max(0, key0 - ctx), c.poison, &c.poisoned);
          ptx::fence_proxy_async_smem();
          __syncwarp();
        }
        ok = tree_wait_warp(&c.p_full[j % C::kP], (uint32_t)(j / C::kP) & 1u, abort_flag);
      } else {
        if (j >= 2) ok = tree_wait_warp(&c.s_empty[j & 1], ((uint32_t)(j - 2) >> 1) & 1u, abort_flag);
        ok = ok && tree_wait_warp(&c.k_full[s], (uint32_t)(j / C::kRingK) & 1u, abort_flag);
      }
      if (!ok) break;
      ptx::tc_fence_after();
      if (ptx::elect_one()) {
        const uint32_t d = tmem_base + (pv ? (uint32_t)C::kColO : (uint32_t)(j & 1) * N);
        const uint32_t t = ring_lo + (uint32_t)s * (C::kSlot >> 4);
        const int nk = pv ? (valid_keys(j) + (Q8 ? 31 : 15)) / (Q8 ? 32 : 16) : Q8 ? 4 : 8;
        if (Q8) {
#pragma unroll
          for (int part = 0; part < 3; ++part) {
            if (!pv && part == 2) break;
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) {
              if (kk >= nk) break;
              tree_umma<Q8>(d, t + kk * 2, a_hi, b_lo + (pv && j % C::kP ? C::kPTile >> 4 : 0) + part * b_half + kk * b_step, b_hi, part ? idesc_lo : idesc,
                            (kk > 0 || part > 0 || (pv && j > 0)) ? 1u : 0u);
            }
          }
        } else {
#pragma unroll
          for (int kk = 0; kk < 8; ++kk) {
            if (kk >= nk) break;
            const uint32_t k4 = (uint32_t)(kk & 3), half = (uint32_t)(kk >> 2);
            tree_umma<Q8>(d, t + half * (kSub >> 4) + k4 * 2u, a_hi, b_lo + half * b_half + k4 * b_step, b_hi, idesc, (kk > 0 || (pv && j > 0)) ? 1u : 0u);
          }
        }
        ptx::umma_commit(pv ? &c.v_empty[s] : &c.k_empty[s]);
        ptx::umma_commit(pv ? &c.p_empty[j % C::kP] : &c.s_full[j & 1]);
      }
      __syncwarp();
    }
  } else if (Q8 && warp == 3) {
    // ---------------- factors of the keys, two tiles ahead of the softmax: each once and not by every group of warps, and the
    // scales' way from memory is nobody's wait ----------------
    for (int j = 0; j < T; ++j) {
      float4 f[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float v_sc = vs[i] < 7.8886091e-31f ? 7.8886091e-31f : vs[i];   // 2^-100 (a row of zeros may come with a scale of 0: it counts in the sum)
        f[i] = make_float4(ks[i] * a.scale_log2, tree_lg2(v_sc), v_sc <= 3.402823466e38f ? tree_rcp(v_sc) * 0x1p-11f : 0.f, 0.f);
      }
      if (j + 1 < T) load_scales(j + 1);
      if (j >= 2 && !tree_wait_warp(&c.s_empty[j & 1], ((uint32_t)(j - 2) >> 1) & 1u, abort_flag)) break;
#pragma unroll
      for (int i = 0; i < 4; ++i) c.key[j & 1][32 * i + lane] = f[i];
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(&c.s_full[j & 1]);
    }
  } else if (warp >= 4) {
    // ---------------- softmax: one thread per key of the tile, 16 lines ----------------
    constexpr int CW = C::kLines, QN = CW / 16;     // lines, and chunks of 16 of them
    const int quarter = warp & 3, group = (warp - 4) >> 2, key = quarter * 32 + lane, col0 = group * CW;
    const uint32_t t_lane = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)col0;
    const int bar = 1 + group;                      // named barrier of the group's four warps
    // this key's row of P: 16-byte pieces of 16 (8) lines, exchanged by the swizzle of rows of 32, 64 or 128 bytes
    const uint32_t p_row = ptx::smem_u32(Ps) + (uint32_t)(key * C::kPRow);
    const int p_turn = C::kPRow == 128 ? key & 7 : C::kPRow == 64 ? (key >> 1) & 3 : (key >> 2) & 1;
    auto p_piece = [&](int q, int i) {              // piece i of chunk q
      const int block = group * QN + q;
      if (Q8) return p_row + (uint32_t)((block ^ p_turn) << 4);
      return p_row + (uint32_t)(N == 128 ? (block >> 2) * 128 * 128 : 0) + (uint32_t)((((N == 128 ? block & 3 : block) * 2 + i) ^ p_turn) << 4);
    };
    ptx::f32x2 acc[QN][8];        // the lines' sums over this thread's keys
#pragma unroll
    for (int i = 0; i < QN * 8; ++i) acc[i / 8][i % 8] = 0ull;
    // the exponents of P from the scores of 16 lines, -infinity where a line does not see the key
    auto exponents = [&](float (&v)[16], int col, float mul, float lv, uint32_t sees) {
      const ptx::f32x2 off2 = ptx::f2_pack(lv + kUp, lv + kUp), mul2 = ptx::f2_pack(mul, mul);
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const ulonglong2 m2 = *reinterpret_cast<const ulonglong2*>(&c.nm[col + i]);
        ptx::f32x2 s0 = ptx::f2_pack(v[i], v[i + 1]), s1 = ptx::f2_pack(v[i + 2], v[i + 3]);
        if (Q8) {
          const ulonglong2 rs = *reinterpret_cast<const ulonglong2*>(&c.rs[col + i]);
          s0 = ptx::f2_mul(s0, rs.x); s1 = ptx::f2_mul(s1, rs.y);
          s0 = ptx::f2_fma(s0, mul2, ptx::f2_add(off2, m2.x)); s1 = ptx::f2_fma(s1, mul2, ptx::f2_add(off2, m2.y));
        } else {
          s0 = ptx::f2_fma(s0, mul2, m2.x); s1 = ptx::f2_fma(s1, mul2, m2.y);
        }
        ptx::f2_unpack(s0, v[i], v[i + 1]);
        ptx::f2_unpack(s1, v[i + 2], v[i + 3]);
      }
      if (sees != 0xffffffffu) {
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = (sees >> i) & 1u ? v[i] : -INFINITY;
      }
    };
    bool ok = true;
    for (int j = 0; j < T; ++j) {
      const int tile = tile0 + j, d = tile - draft0;
      const uint32_t sees = d < 0 ? 0xffffffffu : d == 0 ? seen[0] : d == 1 ? seen[1] : seen[2];
      ok = ok && tree_wait_warp(&c.s_full[j & 1], ((uint32_t)j >> 1) & 1u, abort_flag);
      // (whatever their waits said, the four warps of a group come to its barriers together: a wait that ran out is a no in the
      // vote on the maxima, and the vote behind it ends the loop for all four)
      ptx::tc_fence_after();
      const float4 of_key = Q8 ? c.key[j & 1][key] : make_float4(a.scale_log2, 0.f, 0.f, 0.f);
      const float mul = of_key.x, lv = of_key.y, iv = of_key.z;
      const uint32_t s_col = t_lane + (uint32_t)(j & 1) * N;
      float v[QN][16];
      auto scores = [&]() {
#pragma unroll
        for (int q = 0; q < QN; ++q) ptx::tmem_ld_32x16(s_col + 16 * q, v[q]);
        ptx::tmem_ld_wait();
#pragma unroll
        for (int q = 0; q < QN; ++q) exponents(v[q], col0 + 16 * q, mul, lv, QN == 1 || sees == 0xffffffffu ? sees : (sees >> (16 * q)) | 0xffff0000u);
      };
      bool move = j == 0;      // (there is no maximum yet)
      if (!move) {
        scores();
        float most = -INFINITY;
#pragma unroll
        for (int q = 0; q < QN; ++q)
#pragma unroll
          for (int i = 0; i < 16; i += 2) most = ptx::fmax3(most, v[q][i], v[q][i + 1]);
        move = !ptx::all_agree(bar, 128, ok && !(most > (Q8 ? kHeadE4m3 : kHeadBf16)));
      }
      if (move) {
        // ---- the maxima move: from the scores themselves, over the group's four warps.  Loops over 4 lines that stay
        // loops: this code runs once or a few times, and what it costs is its way from memory ----
#pragma unroll 1
        for (int i = 0; i < CW; i += 4) {
          float u[4];
          tree_tmem_ld4(s_col + i, u);
          ptx::tmem_ld_wait();
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            u[e] = fmaf(Q8 ? u[e] * c.rs[col0 + i + e] : u[e], mul, lv);
            u[e] = tree_max((sees >> (i + e)) & 1u ? u[e] : -INFINITY);
          }
          if (lane == 0) *reinterpret_cast<float4*>(&c.part[quarter][col0 + i]) = make_float4(u[0], u[1], u[2], u[3]);
          __syncwarp();
        }
        if (j > 0)   // O^T: all products so far are in
          ok = ok && tree_wait_warp(&c.p_empty[(j - 1) % C::kP], (uint32_t)((j - 1) / C::kP) & 1u, abort_flag);
        ok = ptx::all_agree(bar, 128, ok);
        if (!ok) break;
        if (quarter == 0 && lane < CW) {
          const int col = col0 + lane;
          const float top = fmaxf(fmaxf(c.part[0][col], c.part[1][col]), fmaxf(c.part[2][col], c.part[3][col]));
          const float old = -c.nm[col], now = fmaxf(top + (Q8 ? kAhead : 0.f), old);
          c.nm[col] = -now;                            // (of columns without a line it stays infinite)
          c.fac[col] = old == -INFINITY ? 0.f : attn_ex2(old - now);
        }
        __syncwarp();
        asm volatile("bar.sync %0, 128;" ::"r"(bar) : "memory");
        if (j > 0) {
#pragma unroll
          for (int i = 0; i < QN * 8; ++i) acc[i / 8][i % 8] = ptx::f2_mul(acc[i / 8][i % 8], *reinterpret_cast<const ptx::f32x2*>(&c.fac[col0 + 2 * i]));
          ptx::tc_fence_after();
#pragma unroll 1
          for (int i = 0; i < CW; i += 4) {
            const uint32_t at = t_lane + (uint32_t)(C::kColO + i);
            const float4 f = *reinterpret_cast<const float4*>(&c.fac[col0 + i]);
            float o[4];
            tree_tmem_ld4(at, o);
            ptx::tmem_ld_wait();
            tree_tmem_st4(at, o[0] * f.x, o[1] * f.y, o[2] * f.z, o[3] * f.w);
          }
          ptx::tmem_st_wait();
          ptx::tc_fence_before();
        }
        scores();
      }
      if (!ok) break;
      ptx::tc_fence_before();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(&c.s_empty[j & 1]);
      auto st16 = [](uint32_t at, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
      };
      uint32_t p[QN][4][Q8 ? 3 : 2];     // of 16 lines, four by four: e4m3 the three parts of them, bf16 two words
      const uint32_t p_at = C::kP == 2 && (j & 1) ? (uint32_t)C::kPTile : 0u;
      auto store = [&](int q) {
        if constexpr (Q8) {
#pragma unroll
          for (int i = 0; i < 3; ++i) st16(p_piece(q, 0) + p_at + i * 128 * C::kPRow, p[q][0][i], p[q][1][i], p[q][2][i], p[q][3][i]);
        } else {
#pragma unroll
          for (int i = 0; i < 2; ++i) st16(p_piece(q, i) + p_at, p[q][2 * i][0], p[q][2 * i][1], p[q][2 * i + 1][0], p[q][2 * i + 1][1]);
        }
      };
      // the P before in this place has been read (a warp whose wait ran out goes on to the next barrier of its group)
      if (C::kTurns) {       // (a half's tile j is behind the other's tile j or j - 1)
        const int team = group * 2 / C::kGroups;
        if (team == 1 || j > 0) ok = tree_wait_warp(&c.turn[team ^ 1], (uint32_t)(j + team - 1) & 1u, abort_flag);
        if (!ok) continue;
      }
      if (C::kP == 2) {
        if (j > 1) ok = tree_wait_warp(&c.p_empty[j & 1], (uint32_t)((j - 2) >> 1) & 1u, abort_flag);
        if (!ok) continue;
      }
      const ptx::f32x2 iv2 = ptx::f2_pack(iv, iv);
#pragma unroll
      for (int q = 0; q < QN; ++q) {
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          const float p0 = attn_ex2(v[q][i]), p1 = attn_ex2(v[q][i + 1]), p2 = attn_ex2(v[q][i + 2]), p3 = attn_ex2(v[q][i + 3]);
          if constexpr (!Q8) {
            acc[q][i / 2] = ptx::f2_add(acc[q][i / 2], ptx::f2_pack(p0, p1));
            acc[q][i / 2 + 1] = ptx::f2_add(acc[q][i / 2 + 1], ptx::f2_pack(p2, p3));
            const __nv_bfloat162 w0 = __floats2bfloat162_rn(p0, p1), w1 = __floats2bfloat162_rn(p2, p3);
            p[q][i / 4][0] = *reinterpret_cast<const uint32_t*>(&w0);
            p[q][i / 4][1] = *reinterpret_cast<const uint32_t*>(&w1);
          } else {
            acc[q][i / 2] = ptx::f2_fma(ptx::f2_pack(p0, p1), iv2, acc[q][i / 2]);
            acc[q][i / 2 + 1] = ptx::f2_fma(ptx::f2_pack(p2, p3), iv2, acc[q][i / 2 + 1]);
            tree_split4(__floats2half2_rn(p0, p1), __floats2half2_rn(p2, p3), p[q][i / 4]);
          }
        }
        if (C::kP == 2) store(q);
      }
      if (C::kP == 1) {
        if (j > 0) ok = tree_wait_warp(&c.p_empty[0], (uint32_t)(j - 1) & 1u, abort_flag);
        if (!ok) continue;
#pragma unroll
        for (int q = 0; q < QN; ++q) store(q);
      }
      ptx::fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(&c.p_full[j % C::kP]);
      if (C::kTurns && lane == 0) ptx::mbar_arrive(&c.turn[group * 2 / C::kGroups]);
    }
    // O^T is complete once the last P has been read
    if (ok) ok = tree_wait_warp(&c.p_empty[(T - 1) % C::kP], (uint32_t)((T - 1) / C::kP) & 1u, abort_flag);
#pragma unroll
    for (int q = 0; q < QN; ++q) {
      float sum[16];
#pragma unroll
      for (int i = 0; i < 8; ++i) ptx::f2_unpack(acc[q][i], sum[2 * i], sum[2 * i + 1]);
      const float part = tree_sum(sum, lane);
      if (lane < 16) c.part[quarter][col0 + 16 * q + lane] = part;
    }
  }
  // ---------------- output ----------------
  __syncthreads();
  const int stretches = a.joined == 1 ? 1 : tree_stretches(a, b);
  const bool failed = c.abort_flag != 0, alone = stretches == 1, apart = !alone && !a.cluster;   // apart: k_tree_join joins them
  // a thread a line: its sum, whether it sees a key that is not finite, its place
  if ((int)threadIdx.x < n) {
    const int col = threadIdx.x, m = line0 + col, r = tree_row(a, m), h = g * G + m - r * G;
    float l = (c.part[0][col] + c.part[1][col]) + (c.part[2][col] + c.part[3][col]);
    bool bad = failed;
    if (c.poisoned)
      for (int w = 0; w < a.words; ++w)
        if (c.poison[w]) bad = bad || (a.mask[((size_t)b * a.max_rows + r) * a.words + w] & c.poison[w]) != 0;
    if (bad) l = __uint_as_float(0x7fffffffu);
    const long long line = (long long)blockIdx.x * a.lines + tree_line(a, b, r, h);
    if (apart) a.part_ml[line] = make_float2(-c.nm[col], l);
    c.rs[col] = l;
    c.fac[col] = !alone ? 1.f : l == 0.f ? 0.f : 1.f / l;      // (NaN stays NaN)
    c.at[col] = apart ? line * kHd : b * a.os[0] + r * a.os[1] + h * a.os[2];
  }
  __syncthreads();
  // O [line][dim] where Q and P were: bf16, or fp32 of a stretch
  if (warp >= 4) {
    const int quarter = warp & 3, col0 = ((warp - 4) >> 2) * C::kLines, ng = min(C::kLines, n - col0), dim = quarter * 32 + lane;
    const uint32_t o_col = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(C::kColO + col0);
    ptx::tc_fence_after();
#pragma unroll 1
    for (int i = 0; i < ng; i += 4) {
      float o[4];
      tree_tmem_ld4(o_col + i, o);        // (whatever is there after a wait that ran out: l is NaN)
      ptx::tmem_ld_wait();
      const float4 f = *reinterpret_cast<const float4*>(&c.fac[col0 + i]);
      const float ff[4] = {f.x, f.y, f.z, f.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (Q8) o[e] *= 0x1p-11f;
        o[e] = ff[e] == 0.f ? 0.f : o[e] * ff[e];
        if (alone) reinterpret_cast<__nv_bfloat16*>(smem_tree)[(col0 + i + e) * kHd + dim] = __float2bfloat16_rn(o[e]);
        else reinterpret_cast<float*>(smem_tree)[(col0 + i + e) * kHd + dim] = o[e];
      }
    }
  }
  __syncthreads();
  if (alone && vec_o) {
    for (int i = threadIdx.x; i < n * 16; i += C::kThreads)
      *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(a.o) + c.at[i >> 4] + (i & 15) * 8) = reinterpret_cast<const uint4*>(smem_tree)[i];
  } else if (alone) {
    for (int i = threadIdx.x; i < n * kHd; i += C::kThreads)
      static_cast<__nv_bfloat16*>(a.o)[c.at[i >> 7] + (i & 127)] = reinterpret_cast<const __nv_bfloat16*>(smem_tree)[i];
  } else if (apart) {
    for (int i = threadIdx.x; i < n * 32; i += C::kThreads)
      *reinterpret_cast<float4*>(a.part_o + c.at[i >> 5] + (i & 31) * 4) = reinterpret_cast<const float4*>(smem_tree)[i];
  }
  if (a.cluster) {
    // the stretches of these lines are the CTAs of the cluster: each joins some of the lines, a warp a line, from the others' shared memory
    // (the barriers want whole warps, and the rows above end inside one)
    __syncwarp();
    ptx::cluster_sync();
    if (!alone) {
      for (int line = (int)blockIdx.x + warp * stretches; line < n; line += C::kThreads / 32 * stretches) {
        float m = -INFINITY, l = 0.f;          // lane = stretch
        if (lane < stretches) {
          m = -tree_remote(&c.nm[line], lane);
          l = tree_remote(&c.rs[line], lane);
        }
        const float top = tree_max(m), w = m == -INFINITY ? 0.f : attn_ex2(m - top);
        l = m == -INFINITY ? l : w * l;        // (NaN without a maximum: a NaN score, or a wait that ran out)
#pragma unroll
        for (int s = 4; s >= 1; s >>= 1) l += __shfl_xor_sync(0xffffffffu, l, s);
        l = __shfl_sync(0xffffffffu, l, 0);
        const float inv = l == 0.f ? 0.f : 1.f / l;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int s = 0; s < stretches; ++s) {
          const float f = __shfl_sync(0xffffffffu, w, s) * inv;
          const float4 p = tree_remote4(smem_tree + line * (kHd * 4) + lane * 16, s);
          o.x = fmaf(f, p.x, o.x); o.y = fmaf(f, p.y, o.y); o.z = fmaf(f, p.z, o.z); o.w = fmaf(f, p.w, o.w);
        }
        const __nv_bfloat162 lo = __floats2bfloat162_rn(o.x, o.y), hi = __floats2bfloat162_rn(o.z, o.w);
        __nv_bfloat16* to = static_cast<__nv_bfloat16*>(a.o) + c.at[line] + lane * 4;
        if (vec_o) {
          *reinterpret_cast<uint2*>(to) = make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
        } else {
          to[0] = lo.x; to[1] = lo.y; to[2] = hi.x; to[3] = hi.y;
        }
      }
    }
    __syncwarp();
    ptx::cluster_sync();      // nobody leaves while another reads its shared memory
  }
  if (loads_k > 0 && c.abort_flag != 0) {
    // given up: what is still on its way lands before another CTA gets this shared memory (with a limit of its own)
    for (int j = max(0, loads_k - C::kRingK); j < loads_k; ++j)
      tree_wait(&c.k_full[j % C::kRingK], (uint32_t)(j / C::kRingK) & 1u, &c.late_flag);
    for (int j = max(0, loads_v - C::kRingV); j < loads_v; ++j)
      tree_wait(&c.v_full[j % C::kRingV], (uint32_t)(j / C::kRingV) & 1u, &c.late_flag);
  }
  if (c.abort_flag != 0 && (warp == 1 || warp == 2)) {
    // ... and what was issued ends before the TMEM that it writes, the shared memory that it reads and the barriers that it arrives on go
    __syncwarp();
    if (ptx::elect_one()) ptx::umma_commit(&c.ended[warp - 1]);
    __syncwarp();
    tree_wait_warp(&c.ended[warp - 1], 0, &c.late_flag);
  }
  ptx::tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    ptx::tc_fence_after();
    ptx::tmem_dealloc(tmem_base, C::kCols);
  }
  if (threadIdx.x == 0 && c.abort_flag && a.status) atomicExch(a.status, DC_ERR_TIMEOUT);
}

}  // namespace dc

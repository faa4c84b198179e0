// What the tensor-core attention kernels share (tc_attn.cuh, tc_attn_few.cuh, tc_tree.cuh).
#pragma once
#include "tc_ptx.cuh"

namespace dc {

constexpr int kHd = 128;
constexpr int kBK = 128;                       // keys per tile
constexpr int kSub = 128 * 128;                // bytes of one [128 rows x 64 bf16] sub-tile

__device__ __forceinline__ float attn_ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// 32 lanes x 16 consecutive 32-bit columns, registers -> TMEM
__device__ __forceinline__ void attn_tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]),
        "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]),
        "r"(r[14]), "r"(r[15])
      : "memory");
}

// Keys of a tile that the P V product takes: its MMAs are 16 keys each, those without a valid key are left out.
__device__ __forceinline__ int attn_pv_keys(int valid) { return (valid + 15) & ~15; }
// Clears what the product takes beyond the valid keys (valid % 16 != 0), in row rr of a V^T tile.  Any tile may
// hold NaN there, a tile of active keys too (the rows of the next sequence, or what an earlier step left), and
// the product with their probability 0 must be 0.  In whole 16-byte pieces, because this is on the serial chain
// of the pass: a Dream-7B prefill of 187 tokens, two tiles of active keys, takes 3836 us like this, 3865 with the
// keys cleared one at a time, and 3823 with active tiles left as they are.
__device__ __forceinline__ void attn_clear_v(uint8_t* tile, int rr, int valid) {
  const int c = valid >> 3, k = valid & 7;   // the piece of eight keys that the valid ones end in, and how many of it are
  auto piece = [&](int i) { return reinterpret_cast<uint4*>(tile + (i >> 3) * kSub + rr * 128 + (((i & 7) ^ (rr & 7)) << 4)); };
  auto kept = [&](int e) { return k > e + 1 ? 0xffffffffu : k > e ? 0xffffu : 0u; };   // of keys e and e + 1
  uint4 w = *piece(c);
  w.x &= kept(0); w.y &= kept(2); w.z &= kept(4); w.w &= kept(6);
  *piece(c) = w;
  if ((c & 1) == 0) *piece(c + 1) = make_uint4(0, 0, 0, 0);
}

// Reduces v[row] over the lanes of a warp, all 32 rows at once: lane i returns row i's result.
template <bool MAX>
__device__ __forceinline__ float few_reduce(float (&v)[32], int lane) {
#pragma unroll
  for (int s = 16; s >= 1; s >>= 1) {
    const bool upper = (lane & s) != 0;
#pragma unroll
    for (int i = 0; i < s; ++i) {
      const float send = upper ? v[i] : v[i + s], keep = upper ? v[i + s] : v[i];
      const float got = __shfl_xor_sync(0xffffffffu, send, s);
      v[i] = MAX ? fmaxf(keep, got) : keep + got;
    }
  }
  return v[0];
}

}  // namespace dc

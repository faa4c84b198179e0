// What the entry points of the operators around a cache share (cache_rows.cu, qk_rope.cu, tree_attn.cu).
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>
#include <stdarg.h>
#include <stdint.h>
#include <stdio.h>

#include "kernels.h"

namespace dc {

inline int op_fail(int code, const char* fmt, ...) {
  char buf[256];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof(buf), fmt, ap);
  va_end(ap);
  set_thread_error(buf);
  return code;
}

// DC_ERR_CUDA where the launch before it failed; the thread's last error is not left behind
inline int op_launched(const char* what) {
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? DC_OK : op_fail(DC_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
}

inline int op_check_cache(const dc_cache* c) {
  if (!c) return op_fail(DC_ERR_INVALID_ARG, "cache is null");
  if (c->dtype != DC_F32 && c->dtype != DC_BF16 && c->dtype != DC_E4M3) return op_fail(DC_ERR_INVALID_ARG, "unknown cache dtype %d", c->dtype);
  if (c->n_layers < 1 || c->max_batch < 1 || c->n_kv_heads < 1 || c->max_ctx < 1) return op_fail(DC_ERR_INVALID_ARG, "cache sizes must be positive");
  if (c->max_ctx % 64) return op_fail(DC_ERR_INVALID_ARG, "max_ctx=%d is not a multiple of 64", c->max_ctx);
  if (c->head_dim < 8 || c->head_dim > 256 || c->head_dim % 8) return op_fail(DC_ERR_UNSUPPORTED, "head_dim=%d is not a multiple of 8 in [8, 256]", c->head_dim);
  if (!c->k || !c->v) return op_fail(DC_ERR_INVALID_ARG, "null cache array");
  if ((c->dtype == DC_E4M3) != (c->k_scale != nullptr) || (c->dtype == DC_E4M3) != (c->v_scale != nullptr))
    return op_fail(DC_ERR_INVALID_ARG, "an e4m3 cache has scales of K and of V, another none");
  return DC_OK;
}

inline int op_check_dtype(const dc_cache* c, int dtype) {
  if (dtype != DC_F32 && dtype != DC_BF16) return op_fail(DC_ERR_INVALID_ARG, "unknown dtype %d of the rows", dtype);
  if (c->dtype != DC_E4M3 && c->dtype != dtype) return op_fail(DC_ERR_UNSUPPORTED, "rows of type %d with a cache of type %d", dtype, c->dtype);
  return DC_OK;
}

inline int op_check_batch(const dc_cache* c, int batch) {
  const int most = c->max_batch < DC_MAX_BATCH ? c->max_batch : DC_MAX_BATCH;
  return batch >= 1 && batch <= most ? DC_OK : op_fail(DC_ERR_SHAPE, "batch %d outside [1, %d]", batch, most);
}

// first[b] + n[b] keys fit the cache, n[b] <= most
inline int op_check_keys(const dc_cache* c, int batch, const int32_t* first, const int32_t* n, int most, const char* what) {
  if (!first || !n) return op_fail(DC_ERR_INVALID_ARG, "null length array");
  for (int b = 0; b < batch; ++b)
    if (first[b] < 0 || n[b] < 0 || n[b] > most || first[b] > c->max_ctx - n[b])
      return op_fail(DC_ERR_SHAPE, "sequence %d: %d keys behind %d (max_ctx %d%s)", b, n[b], first[b], c->max_ctx, what);
  return DC_OK;
}

inline bool op_aligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// DC_OPT_WAIT_LIMIT_US for the waits of dc_tree_attention's kernel; 0 or a CUDA error
int tree_set_wait_limit_us(long long us, cudaStream_t s);
void tree_set_stall(int how);      // DC_OPT_TEST_STALL_TREE

// ---- types --------------------------------------------------------------------------------------------
__device__ __forceinline__ float op_f32(float x) { return x; }
__device__ __forceinline__ float op_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float op_f32(__nv_fp8_e4m3 x) { return (float)x; }
template <typename T> __device__ __forceinline__ T op_to(float x);
template <> __device__ __forceinline__ float op_to<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 op_to<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// the rule of dc_cache for a row whose largest finite magnitude is a
constexpr float kE4m3Max = 448.f;
constexpr float kScaleFloor = 8.271806125530277e-25f;   // 2^-80
__device__ __forceinline__ float op_scale(float a) { return fmaxf(__fdiv_rn(a, kE4m3Max), kScaleFloor); }
__device__ __forceinline__ float op_magnitude(float x) { x = fabsf(x); return x <= 3.402823466e38f ? x : 0.f; }   // (NaN: 0 too)

}  // namespace dc

// dc_cache_write / dc_cache_read: rows of K and V into a cache and back, in 8 bits or as they are.
#include "ops.h"

namespace dc {
namespace {

struct RowsArgs {
  dc_cache c;
  char *k, *v;
  long long ks[5], vs[5];
  int layer, pos[DC_MAX_BATCH], n[DC_MAX_BATCH];
};

// ---- any strides, types and alignment: a warp takes one row of K or V -----------------------------------
// grid (row, sequence * kv head, layer * 2 + side)
constexpr int kAnyWarps = 8;

template <typename T, typename H, bool WRITE>
__global__ void __launch_bounds__(kAnyWarps * 32) k_rows_any(const RowsArgs a) {
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

template <typename T, typename H, bool WRITE>
void launch(const RowsArgs& a, int batch, int n_layers, int most, cudaStream_t s) {
  // (rows beyond the grid are taken in further turns)
  const dim3 grid(min((most + kAnyWarps - 1) / kAnyWarps, 4096), batch * a.c.n_kv_heads, 2 * n_layers);
  k_rows_any<T, H, WRITE><<<grid, kAnyWarps * 32, 0, s>>>(a);
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

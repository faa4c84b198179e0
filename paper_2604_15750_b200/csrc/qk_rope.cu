// dc_qk_norm_rope: norm of each query and key head and its rotation, one pass over the data.
#include <math.h>

#include "ops.h"

namespace dc {
namespace {

struct QkArgs {
  const void *x[2], *gain[2];
  void* y[2];
  long long xs[2][2], ys[2][2];   // row, head
  int heads[2];                   // queries, keys
  const int32_t* pos;
  int rows, hd;
  float eps;
  double freq[128];               // rope_theta^(-2i/hd): radians a position
};

// cos and sin of pos * freq: the product in fp64, brought into one turn there, then fp32
__device__ __forceinline__ void qk_angle(double a, float& c, float& s) {
  const double turns = rint(a * 0.15915494309189535);                            // 1 / (2 pi)
  const double r = fma(-turns, 2.4492935982947064e-16, fma(-turns, 6.283185307179586, a));   // 2 pi in two parts
  sincosf((float)r, &s, &c);
}

// Any head_dim, strides and alignment: a warp takes one head; a lane the pairs lane, lane + 32, ..
constexpr int kQkThreads = 256;

template <typename T>
__global__ void __launch_bounds__(kQkThreads) k_qk_any(const __grid_constant__ QkArgs a) {
  __shared__ float2 turn[128];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, half = a.hd / 2, heads = a.heads[0] + a.heads[1];
  for (int t = blockIdx.x; t < a.rows; t += gridDim.x) {
    __syncthreads();
    const double p = (double)a.pos[t];
    for (int i = threadIdx.x; i < half; i += kQkThreads) qk_angle(p * a.freq[i], turn[i].x, turn[i].y);
    __syncthreads();
    for (int j = blockIdx.y * (kQkThreads / 32) + warp; j < heads; j += gridDim.y * (kQkThreads / 32)) {
      const int w = j >= a.heads[0], h = w ? j - a.heads[0] : j;
      const T* x = static_cast<const T*>(a.x[w]) + t * a.xs[w][0] + h * a.xs[w][1];
      T* y = static_cast<T*>(a.y[w]) + t * a.ys[w][0] + h * a.ys[w][1];
      const T* gain = static_cast<const T*>(a.gain[w]);
      float u[4], v[4], ss = 0.f;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int i = k * 32 + lane;
        u[k] = i < half ? op_f32(x[i]) : 0.f;
        v[k] = i < half ? op_f32(x[i + half]) : 0.f;
        ss = fmaf(u[k], u[k], fmaf(v[k], v[k], ss));
      }
#pragma unroll
      for (int m = 16; m >= 1; m >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, m);
      const float r = rsqrtf(ss / (float)a.hd + a.eps);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int i = k * 32 + lane;
        if (i < half) {
          const float2 cs = turn[i];
          const float p0 = u[k] * r * (gain ? op_f32(gain[i]) : 1.f), p1 = v[k] * r * (gain ? op_f32(gain[i + half]) : 1.f);
          y[i] = op_to<T>(p0 * cs.x - p1 * cs.y);
          y[i + half] = op_to<T>(p1 * cs.x + p0 * cs.y);
        }
      }
    }
  }
}

}  // namespace
}  // namespace dc

extern "C" int dc_qk_norm_rope(const dc_qk_in* in, void* cuda_stream) {
  using namespace dc;
  if (!in) return op_fail(DC_ERR_INVALID_ARG, "null argument");
  if (in->dtype != DC_F32 && in->dtype != DC_BF16) return op_fail(DC_ERR_INVALID_ARG, "unknown dtype %d", in->dtype);
  if (in->rows < 0 || in->n_q_heads < 0 || in->n_kv_heads < 0) return op_fail(DC_ERR_INVALID_ARG, "negative size");
  if (in->n_q_heads > 32768 || in->n_kv_heads > 32768) return op_fail(DC_ERR_UNSUPPORTED, "more than 32768 heads");
  if (in->head_dim < 2 || in->head_dim > 256 || in->head_dim % 2) return op_fail(DC_ERR_UNSUPPORTED, "head_dim=%d is not an even number in [2, 256]", in->head_dim);
  if (!(in->eps >= 0.f) || !(in->rope_theta > 0.f) || isinf(in->eps) || isinf(in->rope_theta)) return op_fail(DC_ERR_INVALID_ARG, "eps must be >= 0 and rope_theta > 0");
  if (in->rows == 0 || in->n_q_heads + in->n_kv_heads == 0) return DC_OK;
  if (!in->pos || (in->n_q_heads && (!in->q || !in->q_out)) || (in->n_kv_heads && (!in->k || !in->k_out)))
    return op_fail(DC_ERR_INVALID_ARG, "null argument");
  QkArgs a;
  a.x[0] = in->q; a.x[1] = in->k; a.gain[0] = in->q_gain; a.gain[1] = in->k_gain; a.y[0] = in->q_out; a.y[1] = in->k_out;
  for (int i = 0; i < 2; ++i) {
    a.xs[0][i] = in->q_stride[i]; a.xs[1][i] = in->k_stride[i];
    a.ys[0][i] = in->q_out_stride[i]; a.ys[1][i] = in->k_out_stride[i];
  }
  a.heads[0] = in->n_q_heads; a.heads[1] = in->n_kv_heads;
  a.pos = in->pos; a.rows = in->rows; a.hd = in->head_dim; a.eps = in->eps;
  const double step = pow((double)in->rope_theta, -2.0 / in->head_dim);
  double f = 1.0;
  for (int i = 0; i < 128; ++i) { a.freq[i] = f; f *= step; }   // (off by at most i roundings of 2^-53)
  const int heads = a.heads[0] + a.heads[1];
  const int across = (heads + kQkThreads / 32 - 1) / (kQkThreads / 32);
  // few rows: the heads of a row spread over CTAs
  const dim3 grid(min(in->rows, 1 << 20), min(across, max(1, 296 / min(in->rows, 296))));
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  if (in->dtype == DC_F32) k_qk_any<float><<<grid, kQkThreads, 0, s>>>(a);
  else k_qk_any<__nv_bfloat16><<<grid, kQkThreads, 0, s>>>(a);
  return op_launched("dc_qk_norm_rope");
}

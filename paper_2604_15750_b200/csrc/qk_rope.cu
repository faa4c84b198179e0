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

// head_dim 64, 128 or 256 on 16-byte boundaries: LPH = head_dim / 16 lanes take a head, each 8 pairs (8 dims of the first
// half, 8 of the second), so that the rotation stays in the lane and the sum of squares takes log2(LPH) shuffles.  A CTA takes a row's
// heads; their loads are under way while its threads make the row's cos and sin.
constexpr int kQkVecThreads = 512;

__device__ __forceinline__ void qk_load(const float* p, float (&x)[8]) {
  const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
  x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
__device__ __forceinline__ void qk_load(const __nv_bfloat16* p, float (&x)[8]) {
  const uint4 w = *reinterpret_cast<const uint4*>(p);
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(u[i] << 16); x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u); }
}
template <typename T> __device__ __forceinline__ void qk_wide(const uint4* w, float (&x)[8]);
template <> __device__ __forceinline__ void qk_wide<float>(const uint4* w, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    x[4 * i] = __uint_as_float(w[i].x); x[4 * i + 1] = __uint_as_float(w[i].y); x[4 * i + 2] = __uint_as_float(w[i].z); x[4 * i + 3] = __uint_as_float(w[i].w);
  }
}
template <> __device__ __forceinline__ void qk_wide<__nv_bfloat16>(const uint4* w, float (&x)[8]) {
  const uint32_t u[4] = {w->x, w->y, w->z, w->w};
#pragma unroll
  for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(u[i] << 16); x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u); }
}
__device__ __forceinline__ void qk_store(float* p, const float (&x)[8]) {
  reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
}
__device__ __forceinline__ void qk_store(__nv_bfloat16* p, const float (&x)[8]) {
  uint32_t u[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 b = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
    u[i] = *reinterpret_cast<const uint32_t*>(&b);
  }
  *reinterpret_cast<uint4*>(p) = make_uint4(u[0], u[1], u[2], u[3]);
}

// Units of work are a row and as many of its heads as the CTA has places; a CTA takes every gridDim.x-th one.  The loads of the next
// unit and its cos and sin are under way while one is worked on.
template <typename T, int HD>
__global__ void __launch_bounds__(kQkVecThreads, 2) k_qk_vec(const __grid_constant__ QkArgs a, const int passes) {
  constexpr int LPH = HD / 16, HALF = HD / 2, W = sizeof(T) / 2;      // 16-byte pieces of a lane's half
  __shared__ __align__(16) float cs[2][HALF], sn[2][HALF];
  const int c = threadIdx.x % LPH * 8, slots = blockDim.x / LPH, heads = a.heads[0] + a.heads[1];
  const long long units = (long long)a.rows * passes;
  uint4 next[2 * W];
  auto load = [&](long long u) {
    const int t = passes == 1 ? (int)u : (int)(u / passes), j = (int)(u - (long long)t * passes) * slots + threadIdx.x / LPH;
    if (j < heads) {
      const int w = j >= a.heads[0];
      const T* x = static_cast<const T*>(a.x[w]) + t * a.xs[w][0] + (w ? j - a.heads[0] : j) * a.xs[w][1] + c;
#pragma unroll
      for (int i = 0; i < W; ++i) { next[i] = reinterpret_cast<const uint4*>(x)[i]; next[W + i] = reinterpret_cast<const uint4*>(x + HALF)[i]; }
    }
  };
  auto angles = [&](long long u, int k) {
    const int t = passes == 1 ? (int)u : (int)(u / passes);
    const double p = (double)a.pos[t];
    for (int i = threadIdx.x; i < HALF; i += blockDim.x) qk_angle(p * a.freq[i], cs[k][i], sn[k][i]);
  };
  load(blockIdx.x);
  angles(blockIdx.x, 0);
  int k = 0;
  for (long long unit = blockIdx.x; unit < units; unit += gridDim.x, k ^= 1) {
    __syncthreads();         // (the table of this unit is there, that of the one before has been read)
    float u[8], v[8];
    qk_wide<T>(next, u);
    qk_wide<T>(next + W, v);
    if (unit + gridDim.x < units) {
      load(unit + gridDim.x);
      angles(unit + gridDim.x, k ^ 1);
    }
    const int t = passes == 1 ? (int)unit : (int)(unit / passes), j = (int)(unit - (long long)t * passes) * slots + threadIdx.x / LPH;
    // (every lane stays for the sums: the lanes of a head may share a warp with those of a head that is not there)
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) ss = fmaf(u[i], u[i], fmaf(v[i], v[i], ss));
#pragma unroll
    for (int m = LPH / 2; m >= 1; m >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, m);
    if (j >= heads) continue;
    const int w = j >= a.heads[0];
    const float r = rsqrtf(ss * (1.f / HD) + a.eps);
    float y0[8], y1[8];
    if (a.gain[w]) {
      const T* gain = static_cast<const T*>(a.gain[w]);
      qk_load(gain + c, y0);
      qk_load(gain + HALF + c, y1);
#pragma unroll
      for (int i = 0; i < 8; ++i) { u[i] *= r * y0[i]; v[i] *= r * y1[i]; }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) { u[i] *= r; v[i] *= r; }
    }
    float cc[8];
    qk_load(cs[k] + c, cc);
#pragma unroll
    for (int i = 0; i < 8; ++i) { y0[i] = u[i] * cc[i]; y1[i] = v[i] * cc[i]; }
    qk_load(sn[k] + c, cc);
#pragma unroll
    for (int i = 0; i < 8; ++i) { y0[i] = fmaf(-v[i], cc[i], y0[i]); y1[i] = fmaf(u[i], cc[i], y1[i]); }
    T* y = static_cast<T*>(a.y[w]) + t * a.ys[w][0] + (w ? j - a.heads[0] : j) * a.ys[w][1];
    qk_store(y + c, y0);
    qk_store(y + HALF + c, y1);
  }
}

template <typename T, int HD>
void launch_vec(const QkArgs& a, cudaStream_t s) {
  constexpr int LPH = HD / 16;
  const int heads = a.heads[0] + a.heads[1];
  // Few rows: the heads of a row are spread over CTAs of a warp or more each, as long as there are SMs without work
  const int spread = max(1, 148 / a.rows);
  const int threads = min(kQkVecThreads, ((heads + spread - 1) / spread * LPH + 31) / 32 * 32);
  const int passes = (heads * LPH + threads - 1) / threads;
  const long long units = (long long)a.rows * passes, most = 148ll * min(2048 / threads, 2 * kQkVecThreads / threads);
  k_qk_vec<T, HD><<<(int)min(units, most), threads, 0, s>>>(a, passes);
}

template <typename T>
bool launch_vec(const QkArgs& a, cudaStream_t s) {
  constexpr int e16 = 16 / sizeof(T);
  if (a.hd != 64 && a.hd != 128 && a.hd != 256) return false;
  for (int w = 0; w < 2; ++w) {
    if (a.heads[w] == 0) continue;
    if (!op_aligned(a.x[w]) || !op_aligned(a.y[w]) || !op_aligned(a.gain[w])) return false;
    for (int i = 0; i < 2; ++i)
      if (a.xs[w][i] % e16 || a.ys[w][i] % e16) return false;
  }
  if (a.hd == 64) launch_vec<T, 64>(a, s);
  else if (a.hd == 128) launch_vec<T, 128>(a, s);
  else launch_vec<T, 256>(a, s);
  return true;
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
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  if (in->dtype == DC_F32 ? launch_vec<float>(a, s) : launch_vec<__nv_bfloat16>(a, s)) return op_launched("dc_qk_norm_rope");
  const int heads = a.heads[0] + a.heads[1];
  const int across = (heads + kQkThreads / 32 - 1) / (kQkThreads / 32);
  // few rows: the heads of a row spread over CTAs
  const dim3 grid(min(in->rows, 1 << 20), min(across, max(1, 296 / min(in->rows, 296))));
  if (in->dtype == DC_F32) k_qk_any<float><<<grid, kQkThreads, 0, s>>>(a);
  else k_qk_any<__nv_bfloat16><<<grid, kQkThreads, 0, s>>>(a);
  return op_launched("dc_qk_norm_rope");
}

// dc_qk_norm_rope: norm of each query and key head and its rotation, one pass over the data.
#include <math.h>

#include <atomic>

#include "ops.h"
#include "pdl.cuh"
#include "tc_ptx.cuh"

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

// cos and sin of a = pos * freq, the product in fp64: there the fraction of a turn is taken (1 / (2 pi) in two parts), the rest is fp32
__device__ __forceinline__ void qk_angle(double a, float& c, float& s) {
  constexpr double inv = 0.15915494309189535, inv_lo = -9.839338337591243e-18;
  const double turn = fma(a, inv_lo, fma(a, inv, -rint(a * inv)));
  sincospif((float)(2.0 * turn), &s, &c);
}

// Any head_dim, strides and alignment: a warp takes one head; a lane the pairs lane, lane + 32, ..
constexpr int kQkThreads = 256;

template <typename T>
__global__ void __launch_bounds__(kQkThreads) k_qk_any(const __grid_constant__ QkArgs a) {
  __shared__ float2 turn[128];
  pdl_trigger();
  pdl_wait();
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
template <typename T> constexpr int kQkVecThreads = sizeof(T) == 4 ? 256 : 512;      // two or three of these CTAs to an SM
template <typename T> constexpr int kQkVecCtas = sizeof(T) == 4 ? 3 : 2;

constexpr int kQkDepth = 4;
__device__ __forceinline__ void qk_copy16(uint4* to, const void* from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(ptx::smem_u32(to)), "l"(from) : "memory");
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

// Bound by HBM: 8152 tokens of 32 + 32 heads, 267 MB, 43.7 us (6.1 TB/s; 45 to 46 where passes go on for a second; fp32 534 MB 125 us,
// 4.3; head_dim 96 by k_qk_any 122 us, 1.7; the same work with the place of every unit calculated
// anew 57 us, as a warp a head 125 us); one token 2.2 us.
// A thread keeps its head (of the CTA's share blockIdx.y) and goes through every gridDim.x-th row.  The loads of the next rows and the
// cos and sin of the next one are under way while a row is worked on.
template <typename T, int HD>
__global__ void __launch_bounds__(kQkVecThreads<T>, kQkVecCtas<T>) k_qk_vec(const __grid_constant__ QkArgs a) {
  constexpr int LPH = HD / 16, HALF = HD / 2, W = sizeof(T) / 2, E16 = 16 / sizeof(T);      // W: 16-byte pieces of a lane's half
  // a row's factors, of queries and of keys: gain and turn in one, y0 = r (u A - v B), y1 = r (v C + u D); a lane's 8 dims are two
  // 16-byte pieces that lie HALF / 8 pieces apart, so that the lanes of a head read neighbouring pieces
  __shared__ __align__(16) float tab[2][2][4][HALF];
  auto place = [](int i) { return ((i >> 2 & 1) * (HALF / 8) + (i >> 3)) * 4 + (i & 3); };
  const int lane = threadIdx.x % LPH, j = blockIdx.y * (blockDim.x / LPH) + threadIdx.x / LPH, w = j >= a.heads[0];
  const bool there = j < a.heads[0] + a.heads[1];
  const int h = there ? (w ? j - a.heads[0] : j) : 0, step = gridDim.x, rows = a.rows;
  const T* x = static_cast<const T*>(a.x[w]) + blockIdx.x * a.xs[w][0] + h * a.xs[w][1] + lane * 8;
  T* y = static_cast<T*>(a.y[w]) + blockIdx.x * a.ys[w][0] + h * a.ys[w][1] + lane * 8;
  const long long x_step = step * a.xs[w][0], y_step = step * a.ys[w][0];
  // this thread's places in a ring of kQkDepth rows: copies that need no registers while they are on their way, and no barrier,
  // because a thread reads what it asked for
  extern __shared__ uint4 qk_ring[];
  uint4* ring = qk_ring + threadIdx.x;
  int loaded = blockIdx.x;
  auto load = [&](int slot) {
    if (there && loaded < rows) {
#pragma unroll
      for (int i = 0; i < W; ++i) {
        qk_copy16(&ring[(slot * 2 * W + i) * blockDim.x], x + i * E16);
        qk_copy16(&ring[(slot * 2 * W + W + i) * blockDim.x], x + HALF + i * E16);
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    x += x_step;
    loaded = loaded < rows - step ? loaded + step : rows;
  };
  // (HALF threads make the factors: their dim's gains and speed stay in registers)
  float g[2][2] = {{1.f, 1.f}, {1.f, 1.f}};
  const int dim = threadIdx.x;
  const double speed = dim < HALF ? a.freq[dim] : 0.0;
  auto gains = [&](int i, float (&to)[2][2]) {
#pragma unroll
    for (int k = 0; k < 2; ++k)
      if (a.gain[k]) {
        to[k][0] = op_f32(static_cast<const T*>(a.gain[k])[i]);
        to[k][1] = op_f32(static_cast<const T*>(a.gain[k])[i + HALF]);
      }
  };
  auto put = [&](int pos, int k, int i, double freq, const float (&gg)[2][2]) {
    float c, s;
    qk_angle((double)pos * freq, c, s);
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      tab[k][q][0][place(i)] = gg[q][0] * c; tab[k][q][1][place(i)] = -gg[q][1] * s;
      tab[k][q][2][place(i)] = gg[q][1] * c; tab[k][q][3][place(i)] = gg[q][0] * s;
    }
  };
  auto factors = [&](int pos, int k) {
    if (dim < HALF) put(pos, k, dim, speed, g);
    for (int i = dim + blockDim.x; i < HALF; i += blockDim.x) {    // (a CTA of fewer threads than pairs: few rows)
      float more[2][2] = {{1.f, 1.f}, {1.f, 1.f}};
      gains(i, more);
      put(pos, k, i, a.freq[i], more);
    }
  };
  pdl_trigger();
  pdl_wait();
#pragma unroll
  for (int i = 0; i < kQkDepth - 1; ++i) load(i);
  if (dim < HALF) gains(dim, g);
  int t = blockIdx.x;
  factors(a.pos[t], 0);
  int k = 0, slot = 0, pos = t < rows - step ? a.pos[t + step] : 0;
  while (true) {
    asm volatile("cp.async.wait_group %0;" ::"n"(kQkDepth - 2) : "memory");
    __syncthreads();         // (the factors of this row are there, those of the one before have been read)
    float u[8], v[8];
    uint4 raw[2 * W];
#pragma unroll
    for (int i = 0; i < 2 * W; ++i) raw[i] = ring[(slot * 2 * W + i) * blockDim.x];
    qk_wide<T>(raw, u);
    qk_wide<T>(raw + W, v);
    load(slot == 0 ? kQkDepth - 1 : slot - 1);      // (the slot of the row before)
    slot = slot == kQkDepth - 1 ? 0 : slot + 1;
    const bool more = t < rows - step;
    if (more) {
      t += step;
      factors(pos, k ^ 1);
      if (t < rows - step) pos = a.pos[t + step];
    }
    // (every lane stays for the sums: the lanes of a head may share a warp with those of a head that is not there)
    ptx::f32x2 u2[4], v2[4], ss2 = 0ull;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      u2[i] = ptx::f2_pack(u[2 * i], u[2 * i + 1]);
      v2[i] = ptx::f2_pack(v[2 * i], v[2 * i + 1]);
      ss2 = ptx::f2_fma(u2[i], u2[i], ptx::f2_fma(v2[i], v2[i], ss2));
    }
    float ss, ss_odd;
    ptx::f2_unpack(ss2, ss, ss_odd);
    ss += ss_odd;
#pragma unroll
    for (int m = LPH / 2; m >= 1; m >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, m);
    if (there) {
      const float r = rsqrtf(ss * (1.f / HD) + a.eps);
      const ptx::f32x2 r2 = ptx::f2_pack(r, r);
      float y0[8], y1[8];
#pragma unroll
      for (int i = 0; i < 4; i += 2) {
        auto two = [&](int of) { return *reinterpret_cast<const ulonglong2*>(&tab[k][w][of][(i / 2 * (HALF / 8) + lane) * 4]); };
        const ulonglong2 A = two(0), B = two(1), Cc = two(2), D = two(3);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const ptx::f32x2 ur = ptx::f2_mul(u2[i + e], r2), vr = ptx::f2_mul(v2[i + e], r2);
          const ptx::f32x2 p = ptx::f2_fma(ur, e ? A.y : A.x, ptx::f2_mul(vr, e ? B.y : B.x)), q = ptx::f2_fma(vr, e ? Cc.y : Cc.x, ptx::f2_mul(ur, e ? D.y : D.x));
          ptx::f2_unpack(p, y0[2 * (i + e)], y0[2 * (i + e) + 1]);
          ptx::f2_unpack(q, y1[2 * (i + e)], y1[2 * (i + e) + 1]);
        }
      }
      qk_store(y, y0);
      qk_store(y + HALF, y1);
    }
    y += y_step;
    if (!more) break;
    k ^= 1;
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
}

template <typename T, int HD>
void launch_vec(const QkArgs& a, cudaStream_t s) {
  constexpr int LPH = HD / 16;
  const int heads = a.heads[0] + a.heads[1];
  // Few rows: the heads of a row are spread over CTAs of a warp or more each, as long as there are SMs without work
  const int spread = max(1, 148 / a.rows);
  const int threads = min(kQkVecThreads<T>, ((heads + spread - 1) / spread * LPH + 31) / 32 * 32);
  const int passes = (heads * LPH + threads - 1) / threads, most = 148 * (kQkVecCtas<T> * kQkVecThreads<T> / threads);
  const int smem = kQkDepth * sizeof(T) * 16 * threads;
  static std::atomic<unsigned long long> done;
  int dev = 0;
  cudaGetDevice(&dev);
  const unsigned long long bit = dev < 64 ? 1ull << dev : 0ull;
  if (!(done.load(std::memory_order_acquire) & bit) &&
      cudaFuncSetAttribute(k_qk_vec<T, HD>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(kQkDepth * sizeof(T) * 16 * kQkVecThreads<T>)) == cudaSuccess)
    done.fetch_or(bit, std::memory_order_release);
  launch_chained(k_qk_vec<T, HD>, dim3(min(a.rows, max(1, most / passes)), passes), dim3(threads), smem, s, a);
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
  a.x[0] = in->q; a.x[1] = in->k; a.y[0] = in->q_out; a.y[1] = in->k_out;
  a.gain[0] = in->n_q_heads ? in->q_gain : nullptr; a.gain[1] = in->n_kv_heads ? in->k_gain : nullptr;   // (not looked at without heads)
  for (int i = 0; i < 2; ++i) {
    a.xs[0][i] = in->q_stride[i]; a.xs[1][i] = in->k_stride[i];
    a.ys[0][i] = in->q_out_stride[i]; a.ys[1][i] = in->k_out_stride[i];
  }
  a.heads[0] = in->n_q_heads; a.heads[1] = in->n_kv_heads;
  a.pos = in->pos; a.rows = in->rows; a.hd = in->head_dim; a.eps = in->eps;
  // (products of up to 127 factors: in the 64 bits of a long double they are off by 2^-57, in a double by 2^-46, which are 2e-6 of a
  // radian at position 2^31)
  const long double step = powl((long double)in->rope_theta, -2.0L / in->head_dim);
  long double f = 1.0L;
  for (int i = 0; i < 128; ++i) { a.freq[i] = i < in->head_dim / 2 ? (double)f : 0.0; f *= step; }
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  if (in->dtype == DC_F32 ? launch_vec<float>(a, s) : launch_vec<__nv_bfloat16>(a, s)) return op_launched("dc_qk_norm_rope");
  const int heads = a.heads[0] + a.heads[1];
  const int across = (heads + kQkThreads / 32 - 1) / (kQkThreads / 32);
  // few rows: the heads of a row spread over CTAs
  const dim3 grid(min(in->rows, 1 << 20), min(across, max(1, 296 / min(in->rows, 296))));
  if (in->dtype == DC_F32) launch_chained(k_qk_any<float>, grid, dim3(kQkThreads), 0, s, a);
  else launch_chained(k_qk_any<__nv_bfloat16>, grid, dim3(kQkThreads), 0, s, a);
  return op_launched("dc_qk_norm_rope");
}

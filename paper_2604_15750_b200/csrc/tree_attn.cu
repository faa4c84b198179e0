// dc_tree_attention: checks, the split into units, launches.
#include "tc.h"
#include "tc_tree.cuh"

#include <atomic>

namespace dc {
namespace {

int sm_count() {
  // (a property of the device; 148 on a B200)
  static std::atomic<int> n[64];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) { cudaGetLastError(); return 148; }
  int v = dev < 64 ? n[dev].load(std::memory_order_relaxed) : 0;
  if (v == 0) {
    if (cudaDeviceGetAttribute(&v, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) { cudaGetLastError(); v = 148; }
    if (dev < 64) n[dev].store(v, std::memory_order_relaxed);
  }
  return v;
}

// once per device and kernel: shared memory beyond 48 KB
template <typename K>
bool opt_in(K kernel, int bytes, std::atomic<unsigned long long>& done) {
  int dev = 0;
  cudaGetDevice(&dev);
  const unsigned long long bit = dev < 64 ? 1ull << dev : 0ull;
  if (done.load(std::memory_order_acquire) & bit) return true;
  // (two CTAs on an SM, in clusters too, want all of its shared memory)
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess ||
      cudaFuncSetAttribute(kernel, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared) != cudaSuccess) return false;
  done.fetch_or(bit, std::memory_order_release);
  return true;
}
template <int N, bool Q8>
bool opt_in_tc() {
  static std::atomic<unsigned long long> done;
  return opt_in(k_tree_tc<N, Q8>, TreeTc<N, Q8>::kSmem, done);
}

// CTAs of k_tree_tc that run at once in clusters of `size`: an SM without enough free neighbours in its part of the device
// gets none (a property of the device)
constexpr int kMaxCluster = 8;
template <int N, bool Q8>
int cluster_slots(int size) {
  using C = TreeTc<N, Q8>;
  static std::atomic<int> known[64][kMaxCluster + 1];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) { cudaGetLastError(); dev = 64; }
  int v = dev < 64 ? known[dev][size].load(std::memory_order_relaxed) : 0;
  if (v == 0) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(size); cfg.blockDim = dim3(C::kThreads); cfg.dynamicSmemBytes = C::kSmem;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = size; attr.val.clusterDim.y = 1; attr.val.clusterDim.z = 1;
    cfg.attrs = &attr; cfg.numAttrs = 1;
    if (!opt_in_tc<N, Q8>() || cudaOccupancyMaxActiveClusters(&v, k_tree_tc<N, Q8>, &cfg) != cudaSuccess || v < 1) {
      cudaGetLastError();
      v = sm_count() / size;
    }
    // (it counts one CTA an SM; where two have room, they do run: 256 CTAs of pairs took one round)
    v = v < 1 ? size : v * size * C::kResident;
    v = v > sm_count() * C::kResident ? sm_count() * C::kResident : v;
    if (dev < 64) known[dev][size].store(v, std::memory_order_relaxed);
  }
  return v;
}

// Units of one call: stretches of `tiles` tiles of keys, `line_tiles` stretches of lines a sequence.
struct TreePlan {
  enum Kind { kTc, kFast, kAny } kind;     // k_tree_tc, k_tree_simt_hd, k_tree_simt
  int shape;                 // lines of a unit
  int tiles, joined, line_tiles, cluster;
  int lines, base[DC_MAX_BATCH];
  uint64_t bytes;
  long long cost;
};

// What units of one kernel take, in 10 ns, measured where K and V come from L2: a tile of 128 keys and the rest of a unit (barriers,
// queries, the first loads' way, the output), with every place of the SMs taken and with one unit an SM; and what it takes more as a
// CTA of a cluster.  kCost64 and kCost128 are of fp32 caches; bf16 and e4m3 ones, which take the same kernel with a conversion on the
// way, go by them too
struct TreeCost { int lines, resident, tile, rest, tile_alone, rest_alone, cluster; };
constexpr TreeCost kCost8[3] = {{32, 2, 125, 450, 92, 310, 100}, {64, 1, 101, 470, 101, 470, 350}, {128, 1, 160, 790, 160, 790, 500}};
constexpr TreeCost kCost16[3] = {{32, 1, 67, 250, 67, 250, 100}, {64, 1, 74, 350, 74, 350, 350}, {128, 1, 128, 660, 128, 660, 500}};
constexpr TreeCost kCost64[3] = {{8, 3, 870, 30, 760, 30, 0}, {32, 2, 980, 230, 950, 200, 0}, {64, 2, 1744, 610, 1680, 570, 0}};    // k_tree_simt_hd
constexpr TreeCost kCost128[3] = {{8, 3, 1640, 50, 1430, 30, 0}, {32, 2, 1820, 420, 1750, 390, 0}, {64, 1, 2535, 770, 2535, 770, 0}};
constexpr TreeCost kCostAny = {kTreeLines, 2, 2000, 500, 2000, 500, 0};
// k_tree_join: a launch, and 1.3 ns for a stretch of a line
constexpr int kJoinLaunch = 300, kJoinLines8 = 8;

// The stretch that ends first: units of about the mean length in rounds of as many as run at once, but not before the longest one
// and not before the keys have come from memory.  (20 drawn calls over e4m3, each with up to 21 forced widths and stretches: what this picks
// takes 1.01 times the best in the mean, 1.12 at worst; 64 to 128 lines over e4m3 took up to 1.8 times as long without the clusters' places
// and the cost of joining.)
template <typename Slots>
TreePlan make_plan(const dc_cache* c, const dc_tree_in* in, const TreeCost& k, TreePlan::Kind kind, Slots in_clusters) {
  TreePlan p{};
  p.shape = k.lines; p.kind = kind; p.cost = -1;
  const int G = in->n_q_heads / c->n_kv_heads, sms = sm_count();
  int longest = 0, units[DC_MAX_BATCH], tiles[DC_MAX_BATCH];
  long long all = 0;
  for (int b = 0; b < in->batch; ++b) {
    const int R = in->n_rows[b];
    p.base[b] = p.lines;
    p.lines += R * in->n_q_heads;
    const int lt = (R * G + k.lines - 1) / k.lines;
    p.line_tiles = p.line_tiles > lt ? p.line_tiles : lt;
    units[b] = lt * c->n_kv_heads;
    tiles[b] = R ? (in->ctx_len[b] + R + kTreeTile - 1) / kTreeTile : 0;
    longest = longest > tiles[b] ? longest : tiles[b];
    all += tiles[b];
  }
  const long long kb = (long long)c->head_dim * (c->dtype == DC_F32 ? 4 : c->dtype == DC_BF16 ? 2 : 1) * 2 * kTreeTile >> 10;   // of a tile
  const long long memory = all * c->n_kv_heads * kb / 65 + k.rest_alone;   // 6.5 TB/s: 65 KB in 10 ns
  long long work = 0;
  for (int b = 0; b < in->batch; ++b) work += (long long)units[b] * tiles[b];
  auto rounds = [&](long long n, int slots, int t, int more) {
    const int one_each = slots / k.resident;
    const long long left = n % slots, mean = n <= slots ? (long long)t * k.tile : work * k.tile / n;
    const long long two = mean + k.rest + more, one = mean * k.tile_alone / k.tile + k.rest_alone + more;
    const long long last = left == 0 ? 0 : left <= one_each ? one : one + (two - one) * (left - one_each) / (slots - one_each);
    const long long cost = n / slots * two + last, most = (long long)t * k.tile_alone + k.rest_alone + more;
    return cost > most ? cost : most;
  };
  // (an 8-bit cache's probabilities end 2^-27 below the largest of a stretch: tc_tree.cuh)
  const int fewest = kind == TreePlan::kTc && c->dtype == DC_E4M3 ? (longest + kTreeMostTiles - 1) / kTreeMostTiles : 1;
  for (int s = fewest < 1 ? 1 : fewest, before = 0; s <= longest && (s <= 256 || p.cost < 0); ++s) {
    const int t = (longest + s - 1) / s;
    if (t == before) continue;
    before = t;
    const int stretches = (longest + t - 1) / t;
    long long n = 0;
    for (int b = 0; b < in->batch; ++b) n += (long long)units[b] * ((tiles[b] + t - 1) / t);
    auto take = [&](long long cost, int cluster) {
      cost = (cost > memory ? cost : memory) + cost / 16;      // (of those that wait for memory the one with less else to do)
      if (p.cost < 0 || cost < p.cost) { p.cost = cost; p.tiles = t; p.cluster = cluster; }
    };
    if (stretches > 1 && stretches <= kMaxCluster && kind == TreePlan::kTc) {
      // (behind the first round a cluster waits until its CTAs find places at once: about a third of them stay empty meanwhile)
      const int slots = in_clusters(stretches);
      take(rounds(n, n > slots ? slots - slots / 3 : slots, t, k.cluster), 1);
    }
    take(rounds(n, k.resident * sms, t, 0) + (stretches == 1 ? 0 : kJoinLaunch + (long long)p.lines * stretches / kJoinLines8), 0);
  }
  p.joined = longest ? (longest + p.tiles - 1) / p.tiles : 0;
  if (p.joined > 1 && !p.cluster) {
    const uint64_t n = (uint64_t)p.joined * p.lines;
    p.bytes = n * 8 + (n & 1) * 8 + n * c->head_dim * 4;
  }
  return p;
}

bool simt_fast(const dc_cache* c, const dc_tree_in* in) {
  return (c->head_dim == 64 || (c->head_dim == 128 && in->dtype == DC_F32)) && op_aligned(c->k) && op_aligned(c->v);
}

// Widths in rising order, the next one where the one before has not room for all lines
template <typename Slots0, typename Slots1, typename Slots2>
TreePlan plan_widths(const dc_cache* c, const dc_tree_in* in, const TreeCost (&k)[3], TreePlan::Kind kind, Slots0 s0, Slots1 s1, Slots2 s2) {
  int most = 0;
  for (int b = 0; b < in->batch; ++b) most = most > in->n_rows[b] ? most : in->n_rows[b];
  const int lines = most * (in->n_q_heads / c->n_kv_heads);
  TreePlan best = make_plan(c, in, k[0], kind, s0);
  if (lines > k[0].lines) {
    const TreePlan p = make_plan(c, in, k[1], kind, s1);
    if (p.cost < best.cost) best = p;
  }
  if (lines > k[1].lines) {
    const TreePlan p = make_plan(c, in, k[2], kind, s2);
    if (p.cost < best.cost) best = p;
  }
  return best;
}

template <bool Q8>
TreePlan plan_tc(const dc_cache* c, const dc_tree_in* in) {
  return plan_widths(c, in, Q8 ? kCost8 : kCost16, TreePlan::kTc, cluster_slots<32, Q8>, cluster_slots<64, Q8>, cluster_slots<128, Q8>);
}

TreePlan plan(const dc_cache* c, const dc_tree_in* in) {
  const uint64_t keys = (uint64_t)c->max_batch * c->n_kv_heads * c->max_ctx, dims = (uint64_t)c->max_batch * c->n_kv_heads * kHd;
  if (in->dtype == DC_BF16 && c->head_dim == kHd && op_aligned(c->k) && op_aligned(c->v) && !(keys >> 31) && !(dims >> 31))
    return c->dtype == DC_E4M3 ? plan_tc<true>(c, in) : plan_tc<false>(c, in);
  auto none = [](int) { return 0; };
  if (simt_fast(c, in)) return plan_widths(c, in, c->head_dim == 64 ? kCost64 : kCost128, TreePlan::kFast, none, none, none);
  return make_plan(c, in, kCostAny, TreePlan::kAny, none);
}

int check(const dc_cache* c, const dc_tree_in* in) {
  int rc = op_check_cache(c);
  if (rc != DC_OK) return rc;
  if (!in) return op_fail(DC_ERR_INVALID_ARG, "null argument");
  if ((rc = op_check_dtype(c, in->dtype)) != DC_OK || (rc = op_check_batch(c, in->batch)) != DC_OK) return rc;
  if (in->layer < 0 || in->layer >= c->n_layers) return op_fail(DC_ERR_SHAPE, "layer %d of %d", in->layer, c->n_layers);
  if (in->n_q_heads < 1 || in->n_q_heads % c->n_kv_heads)
    return op_fail(DC_ERR_INVALID_ARG, "%d query heads over %d kv heads", in->n_q_heads, c->n_kv_heads);
  if (in->n_q_heads / c->n_kv_heads > kTreeMaxGroup)     // (tree_row)
    return op_fail(DC_ERR_UNSUPPORTED, "more than %d query heads of a kv head", kTreeMaxGroup);
  if (in->max_rows < 1 || in->max_rows > DC_MAX_WINDOW) return op_fail(DC_ERR_SHAPE, "max_rows=%d outside [1, %d]", in->max_rows, (int)DC_MAX_WINDOW);
  if (!(in->scale >= 0.f) || in->scale > 1e30f) return op_fail(DC_ERR_INVALID_ARG, "scale outside [0, 1e30]");
  if ((rc = op_check_keys(c, in->batch, in->ctx_len, in->n_rows, in->max_rows, ", max_rows bounds the rows")) != DC_OK) return rc;
  for (int b = 0; b < in->batch; ++b)
    if (in->ctx_len[b] + in->n_rows[b] > kTreeMostKeys) return op_fail(DC_ERR_UNSUPPORTED, "sequence %d: more than %d keys", b, kTreeMostKeys);
  if ((long long)in->max_rows * in->n_q_heads > 524288) return op_fail(DC_ERR_UNSUPPORTED, "more than 524288 rows x query heads");
  return DC_OK;
}

int check_grid(const dc_cache* c, const dc_tree_in* in, const TreePlan& p) {
  return c->n_kv_heads <= 65535 && (long long)p.line_tiles * in->batch <= 65535 ? DC_OK : op_fail(DC_ERR_UNSUPPORTED, "more rows x query heads than one call takes");
}

template <typename T, typename H, int HD, int L>
bool launch_simt_hd(const TreeArgs& a, const TreePlan& p, int batch, cudaStream_t s) {
  static std::atomic<unsigned long long> done;
  if (!opt_in(k_tree_simt_hd<T, H, HD, L>, tree_simt_smem_hd(HD, L), done)) return false;
  return launch_chained(k_tree_simt_hd<T, H, HD, L>, dim3(p.joined, a.c.n_kv_heads, batch * p.line_tiles), dim3(kSimtThreads), tree_simt_smem_hd(HD, L), s, a) == cudaSuccess;
}
template <typename T, typename H, int HD>
bool launch_simt_hd(const TreeArgs& a, const TreePlan& p, int batch, cudaStream_t s) {
  return p.shape == 8 ? launch_simt_hd<T, H, HD, 1>(a, p, batch, s) : p.shape == 32 ? launch_simt_hd<T, H, HD, 4>(a, p, batch, s) : launch_simt_hd<T, H, HD, 8>(a, p, batch, s);
}

template <typename T, typename H>
bool launch_simt(const TreeArgs& a, const TreePlan& p, int batch, cudaStream_t s) {
  if (p.kind == TreePlan::kFast) {
    if (a.c.head_dim == 64) return launch_simt_hd<T, H, 64>(a, p, batch, s);
    if constexpr (sizeof(T) == 4) return launch_simt_hd<T, H, 128>(a, p, batch, s);    // (bf16 rows have the tensor cores)
  }
  static std::atomic<unsigned long long> done;
  if (!opt_in(k_tree_simt<T, H>, tree_simt_smem(256), done)) return false;
  return launch_chained(k_tree_simt<T, H>, dim3(p.joined, a.c.n_kv_heads, batch * p.line_tiles), dim3(128), tree_simt_smem(a.c.head_dim), s, a) == cudaSuccess;
}

template <int N, bool Q8>
bool launch_tc(const TreeArgs& a, const TreePlan& p, int batch, int vec_q, int vec_o, cudaStream_t s) {
  using C = TreeTc<N, Q8>;
  if (!opt_in_tc<N, Q8>()) return false;
  CUtensorMap mk, mv;
  const uint64_t heads = (uint64_t)a.c.max_batch * a.c.n_kv_heads;
  if (!tc_map_bytes(&mk, a.c.k, Q8 ? 1 : 2, heads * a.c.max_ctx, kHd) || !tc_map_bytes(&mv, a.c.v, Q8 ? 1 : 2, heads * kHd, a.c.max_ctx)) return false;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(p.joined, a.c.n_kv_heads, batch * p.line_tiles); cfg.blockDim = dim3(C::kThreads); cfg.dynamicSmemBytes = C::kSmem; cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = p.joined; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr; cfg.numAttrs = p.cluster ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, k_tree_tc<N, Q8>, mk, mv, a, vec_q, vec_o) == cudaSuccess;
}

std::atomic<int> tree_stall;      // DC_OPT_TEST_STALL_TREE

}  // namespace

void tree_set_stall(int how) { tree_stall.store(how, std::memory_order_relaxed); }

int tree_set_wait_limit_us(long long us, cudaStream_t s) {
  const unsigned long long ns = (unsigned long long)us * 1000ull;
  cudaError_t e = cudaMemcpyToSymbolAsync(ptx::g_wait_limit_ns, &ns, sizeof(ns), 0, cudaMemcpyHostToDevice, s);
  if (e == cudaSuccess) e = cudaStreamSynchronize(s);
  return (int)e;
}

}  // namespace dc

using namespace dc;

extern "C" int dc_tree_attention_workspace(const dc_cache* cache, const dc_tree_in* in, uint64_t* bytes) {
  const int rc = check(cache, in);
  if (rc != DC_OK) return rc;
  if (!bytes) return op_fail(DC_ERR_INVALID_ARG, "null argument");
  const TreePlan p = plan(cache, in);
  const int fits = check_grid(cache, in, p);
  if (fits == DC_OK) *bytes = p.bytes;
  return fits;
}

extern "C" int dc_tree_attention(const dc_cache* cache, const dc_tree_in* in, void* cuda_stream) {
  int rc = check(cache, in);
  if (rc != DC_OK) return rc;
  if (!in->q || !in->o) return op_fail(DC_ERR_INVALID_ARG, "null argument");
  const TreePlan p = plan(cache, in);
  if (p.lines == 0) return DC_OK;
  if ((rc = check_grid(cache, in, p)) != DC_OK) return rc;
  if (p.bytes && (!in->workspace || !op_aligned(in->workspace) || in->workspace_bytes < p.bytes))
    return op_fail(DC_ERR_INVALID_ARG, "the workspace needs %llu bytes on a 16-byte boundary", (unsigned long long)p.bytes);
  TreeArgs a;
  a.c = *cache;
  const size_t layer = (size_t)in->layer * cache->max_batch * cache->n_kv_heads * cache->max_ctx;   // keys
  const size_t bytes = layer * cache->head_dim * (cache->dtype == DC_F32 ? 4 : cache->dtype == DC_BF16 ? 2 : 1);
  a.c.k = static_cast<char*>(cache->k) + bytes; a.c.v = static_cast<char*>(cache->v) + bytes;
  if (cache->k_scale) { a.c.k_scale += layer; a.c.v_scale += layer; }
  a.q = in->q; a.o = in->o;
  for (int i = 0; i < 3; ++i) { a.qs[i] = in->q_stride[i]; a.os[i] = in->o_stride[i]; }
  a.mask = in->mask; a.max_rows = in->max_rows; a.words = (in->max_rows + 31) / 32;
  a.nq = in->n_q_heads; a.group = in->n_q_heads / cache->n_kv_heads; a.line_tiles = p.line_tiles;
  a.group_inv = (uint32_t)((1ull << 32) / a.group + 1);
  a.scale_log2 = (in->scale > 0.f ? in->scale : 1.f / sqrtf((float)cache->head_dim)) * 1.4426950408889634f;
  a.tiles = p.tiles; a.joined = p.joined; a.cluster = p.cluster; a.lines = p.lines;
  for (int b = 0; b < DC_MAX_BATCH; ++b) {
    a.base[b] = b < in->batch ? p.base[b] : 0;
    a.ctx[b] = b < in->batch ? in->ctx_len[b] : 0;
    a.rows[b] = b < in->batch ? in->n_rows[b] : 0;
  }
  const uint64_t n = (uint64_t)p.joined * p.lines;
  a.part_ml = static_cast<float2*>(in->workspace);
  a.part_o = reinterpret_cast<float*>(static_cast<char*>(in->workspace) + n * 8 + (n & 1) * 8);
  a.status = in->status; a.stall = tree_stall.load(std::memory_order_relaxed);
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  const bool f32 = in->dtype == DC_F32, q8 = cache->dtype == DC_E4M3;
  const int n_lines = p.kind == TreePlan::kTc ? p.shape : 0;
  int vec_q = op_aligned(in->q), vec_o = op_aligned(in->o);
  for (int i = 0; i < 3; ++i) { vec_q = vec_q && in->q_stride[i] % 8 == 0; vec_o = vec_o && in->o_stride[i] % 8 == 0; }
  const bool ok = n_lines == 32 ? (q8 ? launch_tc<32, true>(a, p, in->batch, vec_q, vec_o, s) : launch_tc<32, false>(a, p, in->batch, vec_q, vec_o, s))
                : n_lines == 128 ? (q8 ? launch_tc<128, true>(a, p, in->batch, vec_q, vec_o, s) : launch_tc<128, false>(a, p, in->batch, vec_q, vec_o, s))
                : n_lines == 64 ? (q8 ? launch_tc<64, true>(a, p, in->batch, vec_q, vec_o, s) : launch_tc<64, false>(a, p, in->batch, vec_q, vec_o, s))
                : f32 ? (q8 ? launch_simt<float, __nv_fp8_e4m3>(a, p, in->batch, s) : launch_simt<float, float>(a, p, in->batch, s))
                      : (q8 ? launch_simt<__nv_bfloat16, __nv_fp8_e4m3>(a, p, in->batch, s) : launch_simt<__nv_bfloat16, __nv_bfloat16>(a, p, in->batch, s));
  if (!ok) {
    const cudaError_t e = cudaGetLastError();
    return op_fail(DC_ERR_CUDA, "dc_tree_attention: %s", e == cudaSuccess ? "no tensor map" : cudaGetErrorString(e));
  }
  if (p.joined > 1 && !p.cluster) {
    const dim3 grid(p.lines);
    if (f32) launch_chained(k_tree_join<float>, grid, dim3(256), 0, s, a, in->batch);
    else launch_chained(k_tree_join<__nv_bfloat16>, grid, dim3(256), 0, s, a, in->batch);
  }
  return op_launched("dc_tree_attention");
}

extern "C" int dc_tree_mask(const int32_t* parent, int32_t n, int32_t words, uint32_t* mask) {
  if (!parent || !mask) return op_fail(DC_ERR_INVALID_ARG, "null argument");
  if (n < 0 || n > DC_MAX_WINDOW || words < (n + 31) / 32) return op_fail(DC_ERR_SHAPE, "%d rows with masks of %d words", n, words);
  for (int r = 0; r < n; ++r)
    if (parent[r] < -1 || parent[r] >= r) return op_fail(DC_ERR_INVALID_ARG, "parent[%d]=%d is not an earlier row or -1", r, parent[r]);
  for (int r = 0; r < n; ++r) {
    uint32_t* m = mask + (size_t)r * words;
    for (int w = 0; w < words; ++w) m[w] = parent[r] >= 0 ? mask[(size_t)parent[r] * words + w] : 0u;
    m[r >> 5] |= 1u << (r & 31);
  }
  return DC_OK;
}

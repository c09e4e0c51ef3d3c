// Paged decode attention over a cache in 4 bits (q4_format.cuh), one or a few tokens of
// every request: for request b with context length T, row i of its n last tokens, q head h
// and g = h / G,
//     out[b][i][h] = sum_{j < T - n + 1 + i} softmax_j(scale q[b][i][h] . k_j) v_j,
// k_j and v_j being c s of the codes and scales of the page (or a 16-bit page's values).
//
// Bound: HBM (9/32 of the bytes of 16-bit pages), so the kernel has 3.5 times fewer
// cycles a key than the 16-bit one.  Its work split, merging and prologue are
// decode_mma.cuh's, in shares at either head size; a warp's work on its keys is
// decode_q4.cuh's.
#include "decode_q4.cuh"

namespace gc {
namespace {

using dec::decode_cta;
using dec::Keys4;

// Threads, resident CTAs and stages of shared memory of a variant.
template <int D, int NT>
struct Shape4 {
  static constexpr int kWarps = 8;
  static constexpr int kCtas = decode_ctas(D, 8 * NT);
  static constexpr int kStages = 3;
  static constexpr int kGroups = 1;
  static constexpr int kThreads = 32 * kWarps;
  static constexpr int kHeads = 8 * NT;
  static constexpr int kStride = D + 4;
  static constexpr int kRingBytes = 2 * kStages * dec::Stage4<D>::kBytes;  // of a warp
  static constexpr int kRedFloats =
      kWarps * kHeads * kStride > kWarps * kRingBytes / 4 ? kWarps * kHeads * kStride
                                                          : kWarps * kRingBytes / 4;
  __device__ static int group() { return 0; }
  __device__ static int tid() { return static_cast<int>(threadIdx.x); }
  __device__ static void sync() { __syncthreads(); }
};

template <int D, int NT>
__global__ void __launch_bounds__(Shape4<D, NT>::kThreads, Shape4<D, NT>::kCtas)
    decode_q4_kernel(const __nv_bfloat16* q, const int32_t* block_table, const int32_t* seq_lens,
                     __nv_bfloat16* out, float* ws, DecGeom geo, int32_t* status,
                     int* merge_counters) {
  extern __shared__ __align__(16) uint8_t smem[];
  dependent_begin();
  decode_cta<Shape4<D, NT>, D, NT, false, false, false, Keys4<D, NT>>(
      smem, dec::ByBlock{}, q, block_table, seq_lens, out, ws, geo, status, merge_counters);
}

template <int D, int NT>
gc_status launch(const gc_kv_pool* pool, const DecodeArgs& a, const DecGeom& geo,
                 cudaStream_t stream) {
  using S = Shape4<D, NT>;
  const size_t smem = decode_smem_bytes<S>(a.batch);
  auto kernel = decode_q4_kernel<D, NT>;
  cudaError_t e = cudaSuccess;
  // a block gets 48 KB without asking, its static words (well below 1 KB) included
  if (smem > 47 * 1024)
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             static_cast<int>(smem));
  if (e != cudaSuccess) return cuda_fail(e, a.who);
  const int grid = min(S::kCtas * pool->num_sms, kMergeCounters);
  e = launch_dependent(kernel, grid, S::kThreads, smem, stream,
                       static_cast<const __nv_bfloat16*>(a.q), a.block_table, a.seq_lens,
                       static_cast<__nv_bfloat16*>(a.out), static_cast<float*>(a.workspace), geo,
                       pool->status, pool->merge_counters);
  if (e != cudaSuccess) return cuda_fail(e, a.who);
  return GC_OK;
}

}  // namespace

size_t decode_q4_workspace_bytes(const gc_kv_pool* pool, int32_t num_q_heads, int32_t tokens) {
  return decode_share_bytes(pool->cfg.head_dim, num_q_heads / pool->cfg.num_kv_heads * tokens,
                            pool->num_sms, kMergeCounters);
}

gc_status launch_decode_q4(const gc_kv_pool* pool, const DecodeArgs& a, const Q4Cache& cache,
                           int32_t tokens, cudaStream_t stream) {
  gc_status st = check_decode(pool, a);
  if (st != GC_OK) return st;
  const size_t need = decode_q4_workspace_bytes(pool, a.num_q_heads, tokens);
  if (a.workspace == nullptr || a.workspace_bytes < need)
    return fail(GC_ERR_INVALID_ARG,
                "%s: workspace of %zu bytes needed (gc_paged_decode_q4_workspace_bytes), got %zu",
                a.who, need, a.workspace_bytes);
  // the work is numbered in units of keys with 32-bit ints (decode_units)
  const int64_t cap = static_cast<int64_t>(a.max_blocks) * pool->cfg.page_size;
  const long long units =
      static_cast<long long>(a.batch) * pool->cfg.num_kv_heads * ((cap + 127) / 128);
  if (units + 2LL * pool->num_sms > 2147483647LL)
    return fail(GC_ERR_UNSUPPORTED, "%s: %lld work items", a.who, units);
  DecGeom geo = decode_geom(pool, a, nullptr, nullptr);
  geo.q4_cache = cache.data;
  geo.q4_table = cache.table;
  geo.q4_pages = cache.pages;
  geo.q4_page = static_cast<uint32_t>(
      geo.Hkv * q4_head_bytes(pool->cfg.head_dim, pool->cfg.page_size));
  geo.q4_plane = static_cast<int64_t>(cache.pages) * geo.q4_page;
  geo.tokens = tokens;
  while ((1 << geo.g_shift) < geo.G) ++geo.g_shift;
  const bool narrow = geo.G * tokens <= 8;
  if (pool->cfg.head_dim == 128)
    return narrow ? launch<128, 1>(pool, a, geo, stream) : launch<128, 2>(pool, a, geo, stream);
  return narrow ? launch<64, 1>(pool, a, geo, stream) : launch<64, 2>(pool, a, geo, stream);
}

}  // namespace gc

// Paged decode attention on the register path (mma.sync), bf16 and 8-bit pages.
//
// One new token per request (Sec. 2.1: the decode phase; with the KV cache it
// is bound by memory): for request b with context length T, kv head g and its
// G q heads h,
//     out[b][h] = sum_{j < T} softmax_j(scale * q[b][h] . k_j) v_j.
//
// Bound: HBM (every context key's K and V row read once), as long as nothing
// but the loads sits between memory and the products.  A query has only G rows
// per kv head, so the tensor work is small (mma.sync runs at 2 cycles a product
// and SM here; ncu: tensor pipe 10 % busy) and the products are taken
// transposed with the keys on the 16-row side of mma.m16n8k16:
//     S^T (16 keys x 8 heads)  = K (16 x d) . Q^T (d x 8)
//     O^T (d x 8 heads)       += V^T (d x 16) . P^T (16 x 8)
// The order of d within the products is free, and so is the order of a tile's
// output rows, so both are chosen to make the fragments plain loads: a thread
// reads 32 bytes (bf16) or 16 codes of a key's row, coalesced over the warp,
// and that is its share of the A operand of both products.  K, V and the 8-bit
// codes never pass through shared memory: 8-bit codes are dequantised in the
// registers they arrive in, with the restore's rounding.  (The path before
// this one fed tcgen05 from shared memory; writing the dequantised tiles there
// was most of the 8-bit variant's time.)  P^T comes from S^T by a transposing
// movmatrix.
//
// A warp takes 16 keys at a time (a group: within one page, since pages hold
// at least 16) with its own online softmax: the reference max of a head is the
// first group's, raised (O and the sums rescaled) only when a score exceeds it
// by 2^56.  The warps of a CTA take the groups of a piece in turn and merge at
// its end through shared memory.  Loads of the next group's K are issued when
// this group's K has been consumed, V likewise.
//
// Work split.  Many short contexts (none above 256 keys): one (request, kv
// head) pair per warp, no merging.  Otherwise, head_dim 128: the groups of all
// (request, kv head) pairs, numbered in order and each with an allowance for its
// fixed cost in front, are cut into one equal share per CTA, so every SM is busy
// for the same time whatever the mix of context lengths.  A pair that a share boundary cuts is done in pieces: each writes
// fp32 partials (O^T unscaled, its reference max, its sum) and the last CTA to
// finish one of the pair's pieces combines them (a counter per cut pair in the
// pool's control block).  head_dim 64: key ranges of a fixed number of 128-key
// tiles, dealt to the CTAs in turn; ranges of a request with several write
// partials that the merge kernel (decode.cu) combines.
//
// bf16 and 8-bit pages run the same products in the same order, so decode over
// 8-bit pages equals the 8-bit restore followed by decode bit for bit.
//
// Small calls of shared prefixes and cross attention (kTwo): a row's keys are those of its
// group's (or request's) page list, then its own.  Four requests of 4 q heads and 1 kv head
// of 64 behind 256 tokens take 7 us, of which the kernel's start and end are most.
//
// Measured (one call, back to back; tcgen05 kernel -> this one): 8 contexts of 9216
// keys, 64 q / 8 kv heads of 128, bf16 55.7 -> 52.8 us (5.7 TB/s), 8-bit 85.8 -> 42.7
// us; 64 multi-turn contexts (243k keys) bf16 182 -> 151 us (6.6 TB/s), 8-bit 295 ->
// 120 us; 128 contexts of 12-100 keys 37.4 -> 9.2 us; head_dim 64, 64 multi-turn
// contexts 228 -> 117 us, 5 contexts of 240-1900 keys 17.8 -> 8.1 us, 8-bit 32
// contexts of up to 3000 keys 55.4 -> 41.5 us.  The 8-bit variant is bound by its
// instructions and their latencies (48 % of the issue slots); copies of its codes
// through shared memory two groups ahead and 16 instead of 12 warps an SM did not
// help.
#include "decode_mma.cuh"

namespace gc {
namespace {

using dec::decode_cta;
using dec::Shape;

template <int D, int NT, bool kQ8, bool kParts, bool kTwo>
__global__ void __launch_bounds__(Shape<D, NT>::kThreads, Shape<D, NT>::kCtas)
    decode_mma_kernel(const __nv_bfloat16* q, const int32_t* block_table,
                      const int32_t* seq_lens, __nv_bfloat16* out,
                      float* ws, DecGeom geo, int32_t* status,
                      int* merge_counters) {
  extern __shared__ __align__(16) uint8_t smem[];
  dependent_begin();
  decode_cta<Shape<D, NT>, D, NT, kQ8, kParts, kTwo>(smem, dec::ByBlock{}, q, block_table, seq_lens, out,
                                               ws, geo, status, merge_counters);
}

template <int D, int NT, bool kQ8, bool kParts, bool kTwo>
gc_status launch(const gc_kv_pool* pool, const DecodeArgs& a, const DecGeom& geo, int grid,
                 cudaStream_t stream) {
  using S = Shape<D, NT>;
  const size_t smem = decode_smem_bytes<S>(a.batch, kTwo);
  auto kernel = decode_mma_kernel<D, NT, kQ8, kParts, kTwo>;
  cudaError_t e = cudaSuccess;
  // a block gets 48 KB without asking, its static words (well below 1 KB) included
  if (smem > 47 * 1024) e = allow_shared<decode_smem_bytes<S>(kMaxBatch, kTwo)>(kernel);
  if (e != cudaSuccess) return cuda_fail(e, a.who);
  e = launch_dependent(kernel, grid, S::kThreads, smem, stream,
                       static_cast<const __nv_bfloat16*>(a.q), a.block_table, a.seq_lens,
                       static_cast<__nv_bfloat16*>(a.out), static_cast<float*>(a.workspace), geo,
                       pool->status, pool->merge_counters);
  if (e != cudaSuccess) return cuda_fail(e, a.who);
  return GC_OK;
}

template <int D, bool kQ8, bool kParts = false, bool kTwo = false>
gc_status launch_heads(const gc_kv_pool* pool, const DecodeArgs& a, DecGeom geo, int max_ranges,
                       cudaStream_t stream) {
  const bool narrow = geo.G <= 8;
  const int ctas = narrow ? Shape<D, 1>::kCtas : Shape<D, 2>::kCtas;
  int grid = min(ctas * pool->num_sms, kMergeCounters);
  if (geo.range_tiles) grid = min(grid, max_ranges);
  return narrow ? launch<D, 1, kQ8, kParts, kTwo>(pool, a, geo, grid, stream)
                : launch<D, 2, kQ8, kParts, kTwo>(pool, a, geo, grid, stream);
}

}  // namespace

// (At most one CTA per merge counter of the pool's control block.)
size_t decode_share_workspace_bytes(const gc_kv_pool* pool, int32_t num_q_heads) {
  return decode_share_bytes(pool->cfg.head_dim, num_q_heads / pool->cfg.num_kv_heads,
                            pool->num_sms, kMergeCounters);
}

gc_status launch_decode_mma(const gc_kv_pool* pool, const DecodeArgs& a, const DecodeSplit* split,
                            cudaStream_t stream, const Q8Pages* q8) {
  const auto& cfg = pool->cfg;
  const DecGeom geo = decode_geom(pool, a, split, q8);
  const long long ranges =
      split ? static_cast<long long>(a.batch) * cfg.num_kv_heads * split->splits : 0;
  const int max_ranges = static_cast<int>(ranges < kMergeCounters ? ranges : kMergeCounters);
  const bool two = a.prefix.groups > 0;
  if (cfg.head_dim == 128)
    return two       ? launch_heads<128, false, false, true>(pool, a, geo, max_ranges, stream)
           : a.own.o ? launch_heads<128, false, true>(pool, a, geo, max_ranges, stream)
           : q8      ? launch_heads<128, true>(pool, a, geo, max_ranges, stream)
                     : launch_heads<128, false>(pool, a, geo, max_ranges, stream);
  return two       ? launch_heads<64, false, false, true>(pool, a, geo, max_ranges, stream)
         : a.own.o ? launch_heads<64, false, true>(pool, a, geo, max_ranges, stream)
         : q8      ? launch_heads<64, true>(pool, a, geo, max_ranges, stream)
                   : launch_heads<64, false>(pool, a, geo, max_ranges, stream);
}

}  // namespace gc

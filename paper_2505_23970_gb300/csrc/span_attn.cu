// Cross attention and decode behind a shared prefix on the tensor-core kernels.
//
// Both are attention whose rows see all keys of a page list: a request's new tokens
// over its cached states, or all requests of a group (one token each) over the group's
// shared pages.  The kernels of the prefill attention take them (attn_tc2.cu at
// head_dim 128, attn_tc.cu at 64) without the causal limit, cut where the items alone
// would leave SMs idle (span.cuh); the rows of a group's requests lie next to each
// other, so the shared keys are read once for 256 of them.  The requests' own keys are
// decoded by some of the same kernel's CTAs (or by the decode kernel before it), and small
// calls by the decode kernel alone, row by row (row_by_row).
//
// P is rounded to bf16 for its product, on the tiles and row by row (the tensor cores take it
// with V as it is kept); scores, maxima, sums, O and the pieces are binary32.  Against 64 bits
// the relative error is 0.0020 to 0.0024; the output's rounding alone is 0.0017.
//
// Here: which way a call goes, its workspace, and the joins of pieces.  A join is bound by
// latency: its blocks read the plan, the row's place and then eight pieces at a time
// (pieces one after the other 10 to 37 us, eight together 4 to 8, at 512 to 4096 rows).
#include "gc_internal.cuh"
#include "sm103_ptx.cuh"
#include "span.cuh"

namespace gc {
namespace {

// One row's join over its pieces and, last, another part (m, l, o): four columns of a
// row per thread, eight pieces' loads in flight.
struct Join {
  float M = -INFINITY, L = 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);

  // row `row` of a cut item
  template <int D>
  __device__ __forceinline__ void pieces(const SpanGeom& sp, const SpanCut& cut, int row, int c) {
    constexpr int kBatch = 8;
    for (int s0 = cut.c0; s0 <= cut.c1; s0 += kBatch) {
      float2 ml[kBatch];
      float4 o[kBatch];
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        const int s = s0 + k;
        const int64_t x =
            static_cast<int64_t>(2 * s + (s == cut.c0 ? cut.first : 0)) * sp.stride + row;
        ml[k] = s <= cut.c1 ? ld_plain(sp.ml + x) : make_float2(-INFINITY, 0.f);
        o[k] = s <= cut.c1 ? ld_plain(reinterpret_cast<const float4*>(sp.o + x * D) + c)
                           : make_float4(0.f, 0.f, 0.f, 0.f);
      }
      float Mn = M;
#pragma unroll
      for (int k = 0; k < kBatch; ++k) Mn = fmaxf(Mn, ml[k].x);
      rescale(Mn);
#pragma unroll
      for (int k = 0; k < kBatch; ++k) add(ml[k], o[k]);
    }
  }
  __device__ __forceinline__ void part(const float2& ml, const float4& o) {
    rescale(fmaxf(M, ml.x));
    add(ml, o);
  }
  __device__ __forceinline__ uint2 rounded() const {
    const float inv = L == 0.f ? 0.f : 1.f / L;  // (no key at all)
    return make_uint2(ptx::pack_bf16x2(acc.x * inv, acc.y * inv),
                      ptx::pack_bf16x2(acc.z * inv, acc.w * inv));
  }

 private:
  __device__ __forceinline__ void rescale(float Mn) {
    const float f = M == -INFINITY ? 0.f : ptx::ex2_approx(M - Mn);
    L *= f;
    acc.x *= f;
    acc.y *= f;
    acc.z *= f;
    acc.w *= f;
    M = Mn;
  }
  __device__ __forceinline__ void add(const float2& ml, const float4& o) {
    const float w = ml.x == -INFINITY ? 0.f : ptx::ex2_approx(ml.x - M);
    L = fmaf(ml.y, w, L);
    acc.x = fmaf(o.x, w, acc.x);
    acc.y = fmaf(o.y, w, acc.y);
    acc.z = fmaf(o.z, w, acc.z);
    acc.w = fmaf(o.w, w, acc.w);
  }
};

// Cross attention: the rows of the items that were cut.  Every cut item has one share in
// which it begins and which it is the last of: block (share, row chunk).
template <int D>
__global__ void __launch_bounds__(256)
    cross_join_kernel(SpanGeom sp, __nv_bfloat16* out, int Hq, int G, int* work_counter) {
  dependent_begin();
  constexpr int kLanes = D / 4;  // four columns each
  constexpr int kRowsPerBlock = 256 / kLanes;
  constexpr int kChunks = kSpanRows / kRowsPerBlock;  // of an item
  const int worker = static_cast<int>(blockIdx.x) / kChunks;
  const int chunk = static_cast<int>(blockIdx.x) % kChunks;
  const int share = ld_plain(sp.plan), workers = ld_plain(sp.plan + 1);
  // (a SpanCutItem)
  const int4 x = ld_plain(sp.cuts_at + 2 * worker), y = ld_plain(sp.cuts_at + 2 * worker + 1);
  if (blockIdx.x == 0 && threadIdx.x == 0) *work_counter = 0;  // for the next call
  if (share == 0 || worker >= workers || x.x < 0) return;
  const SpanCut cut{worker, x.x, x.y};
  const int g = x.z, cu = y.x, row = chunk * kRowsPerBlock + static_cast<int>(threadIdx.x) / kLanes;
  const int at = x.w * kSpanRows + row;  // q row of the request and kv head
  if (at >= y.y * G) return;
  const int c = static_cast<int>(threadIdx.x) % kLanes;
  Join j;
  j.pieces<D>(sp, cut, row, c);
  *reinterpret_cast<uint2*>(
      out + (static_cast<int64_t>(cu + at / G) * Hq + g * G + at % G) * D + 4 * c) = j.rounded();
}

// Decode behind a shared prefix: every row of a request that is not skipped.
template <int D>
__global__ void __launch_bounds__(256)
    shared_join_kernel(SpanGeom sp, const int32_t* own_lens, int own_cap, DecodeParts own,
                       __nv_bfloat16* out, int Hq, int G, int64_t rows, int32_t* status,
                       int* work_counter) {
  dependent_begin();
  if (blockIdx.x == 0 && threadIdx.x == 0) *work_counter = 0;  // for the next call
  constexpr int kLanes = D / 4;
  const int c = static_cast<int>(threadIdx.x) % kLanes;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * (256 / kLanes) + threadIdx.x / kLanes;
  if (row >= rows) return;
  const int b = static_cast<int>(row / Hq), h = static_cast<int>(row - static_cast<int64_t>(b) * Hq);
  const int T = ld_plain(own_lens + b), share = ld_plain(sp.plan);
  const int4 p = ld_plain(sp.prior + b);  // SpanPrior
  if (p.z < 0) record_error(status, GC_ERR_OUT_OF_RANGE);
  if (T < 0 || T > own_cap || p.z < 0) return;
  auto load = [&](const DecodeParts& parts, bool any, float2& ml, float4& o) {
    ml = any ? ld_plain(parts.ml + row) : make_float2(-INFINITY, 0.f);
    o = any ? ld_plain(reinterpret_cast<const float4*>(parts.o + row * D) + c)
            : make_float4(0.f, 0.f, 0.f, 0.f);
  };
  float2 ml;
  float4 o;
  load(own, T > 0, ml, o);
  Join j;
  SpanCut cut{0, 0, 0};
  const int g = h / G;
  if (share && p.z > 0) cut = span_cut(p.x + g * span_per(p.z), p.z, share);
  if (cut.c1 > cut.c0) {
    j.pieces<D>(sp, cut, p.w % kSpanRows + (h - g * G), c);
  } else {
    float2 sml;
    float4 so;
    load(sp.whole, p.z > 0, sml, so);
    j.part(sml, so);
  }
  j.part(ml, o);
  *reinterpret_cast<uint2*>(out + row * D + 4 * c) = j.rounded();
}

// Items that may be cut: claimed from the counter that the join behind them leaves at 0.
// Others may have no join: claimed from the one that the launch clears, as a prefill's.
gc_status launch_items(const gc_kv_pool* pool, const AttnArgs& a, const SpanGeom& span,
                       cudaStream_t stream, const OwnDecode* own = nullptr) {
  int* counter = span.cuts ? pool->span_counter : pool->work_counter;
  return pool->cfg.head_dim == 128
             ? launch_attn_tc2(pool, a, stream, counter, nullptr, &span, own)
             : launch_attn_tc_span(pool, a, stream, counter, span, own);
}

// The join behind a call's items.
template <typename... P, typename... A>
gc_status launch_join(const gc_kv_pool* pool, const char* who, void (*join)(P...), int64_t blocks,
                      cudaStream_t stream, A... args) {
  const cudaError_t e =
      launch_dependent(join, static_cast<unsigned>(blocks), 256, 0, stream, args...);
  if (e == cudaSuccess) return GC_OK;
  // (no join to do it)
  cudaMemsetAsync(pool->span_counter, 0, sizeof(int), stream);
  return cuda_fail(e, who);
}

gc_status check_space(const char* who, size_t need, const void* workspace, size_t bytes) {
  if (need == 0 || (workspace && bytes >= need)) return GC_OK;
  return fail(GC_ERR_INVALID_ARG, "%s: workspace of %zu bytes needed, got %zu", who, need,
              workspace ? bytes : 0);
}

}  // namespace

// Small calls are decoded row by row, the shared keys (or states) in front of the row's own
// ones: the keys are then read once for every row, mostly from the L2, but in one launch
// of the decode kernel, without a join and without the start of the tensor-core kernels.
// By the room in the block tables, as the lengths are on the device: rows x `keys` x kv
// heads.  Measured at lengths that fill it, row by row | tiles (us, heads of 128 then 64):
//   shared: 4 requests behind 256 tokens, 1 kv head, 7.0 | 13.7, 7.3 | 11.6; behind 1000
//   tokens with 100 own ones, 8 kv heads, 16 requests 16.0 | 19.4, 13.0 | 16.7, 32 20.7 |
//   19.8, 16.4 | 20.9, 128 56 | 32, 39 | 28; 32 behind 3500 and 100, 4 kv heads, 24.3 |
//   19.5, 18.8 | 20.5;
//   cross: 16 tokens over 1000 states each, 1 kv head, 9.2 | 18.3, 8.2 | 20.6; 12 over
//   1000, 8 kv heads, 13.1 | 18.1, 11.3 | 20.2; 320 over 300, 2 kv heads, 38.6 | 15.3,
//   22.3 | 18.6.  With two steps of keys nothing is cut and tiles take 9 us: 64 over 256,
//   1 kv head, 9.2 | 8.7, 8.1 | 9.2; 2 kv heads, 16.0 | 8.9, 10.1 | 9.2.
static bool row_by_row(const gc_kv_pool* pool, int64_t rows, int64_t keys, bool shared) {
  const bool wide = pool->cfg.head_dim == 128;
  const int64_t most = shared ? (wide ? 262144 : 458752)
                       : keys > 256 ? (wide ? 131072 : 163840) : (wide ? 8192 : 16384);
  return rows <= 8192 && rows * keys * pool->cfg.num_kv_heads <= most;
}

size_t cross_workspace_bytes(const gc_kv_pool* pool, int32_t batch, int32_t max_blocks,
                             int32_t num_q_heads, int32_t total_new_tokens) {
  if (row_by_row(pool, total_new_tokens, static_cast<int64_t>(max_blocks) * pool->cfg.page_size,
                 false))
    return decode_share_workspace_bytes(pool, num_q_heads);
  return span_space(pool, total_new_tokens, batch, max_blocks, num_q_heads, false).end;
}

// The rows of a call one by one; own_lens: nullptr if they have no keys of their own.
static gc_status launch_rows(const gc_kv_pool* pool, const SpanArgs& a, const char* who,
                             const int32_t* own_table, const int32_t* own_lens, int32_t own_blocks,
                             const DecodePrefix& prefix, cudaStream_t stream) {
  DecodeArgs all{a.q, a.out, own_table, own_lens, a.rows, own_blocks, a.layer, a.num_q_heads,
                 a.softmax_scale, a.workspace, a.workspace_bytes, who};
  all.prefix = prefix;
  const gc_status st = check_decode(pool, all);
  return st == GC_OK ? launch_decode_mma(pool, all, nullptr, stream, nullptr) : st;
}

gc_status launch_cross(const gc_kv_pool* pool, const SpanArgs& a, cudaStream_t stream) {
  const char* who = "gc_paged_cross_attn";
  const auto& cfg = pool->cfg;
  gc_status st = check_space(
      who, cross_workspace_bytes(pool, a.batch, a.max_blocks, a.num_q_heads, a.rows), a.workspace,
      a.workspace_bytes);
  if (st != GC_OK) return st;
  if (row_by_row(pool, a.rows, static_cast<int64_t>(a.max_blocks) * cfg.page_size, false))
    return launch_rows(pool, a, who, nullptr, nullptr, 1,
                       DecodePrefix{a.block_table, a.lens, a.start, a.new_lens, a.batch,
                                    a.max_blocks}, stream);
  const SpanSpace space = span_space(pool, a.rows, a.batch, a.max_blocks, a.num_q_heads, false);
  const SpanGeom span = span_geom(space, static_cast<int64_t>(a.max_blocks) * cfg.page_size, false,
                                  a.workspace);
  const AttnArgs args{a.q, a.out, a.block_table, a.lens, a.new_lens, a.start, a.batch,
                      a.max_blocks, a.layer, a.num_q_heads, a.rows, a.softmax_scale, who};
  st = launch_items(pool, args, span, stream);
  if (st != GC_OK || !span.cuts) return st;
  // (one block per share and 1024 / d rows)
  const int chunks = kSpanRows / (1024 / cfg.head_dim);
  const auto join = cfg.head_dim == 128 ? cross_join_kernel<128> : cross_join_kernel<64>;
  return launch_join(pool, who, join, space.slots / 2 * chunks, stream, span,
                     static_cast<__nv_bfloat16*>(a.out), a.num_q_heads,
                     a.num_q_heads / cfg.num_kv_heads, pool->span_counter);
}

// One kernel for both sides of a call, unless the own keys' side needs more registers
// than the span kernel's threads have (16 heads of 128), or the units could not be
// numbered, or two groups an SM not counted.  Otherwise a kernel each.
static bool decodes_in_kernel(const gc_kv_pool* pool, const SpanArgs& a) {
  const auto& cfg = pool->cfg;
  const int64_t G = a.num_q_heads / cfg.num_kv_heads;
  const int64_t items = cfg.num_kv_heads * (a.batch * G / kSpanRows + a.groups);
  const int64_t steps = static_cast<int64_t>(a.max_shared_blocks) * cfg.page_size / 128 + 1;
  const int64_t own = static_cast<int64_t>(a.batch) * cfg.num_kv_heads *
                      (static_cast<int64_t>(a.max_blocks) * cfg.page_size / 128 + 1);
  return own + 2 * kMergeCounters < 2147483647LL && (cfg.head_dim == 64 || G <= 8) &&
         a.groups <= kSpanRequests && 2 * pool->num_sms <= kMergeCounters &&
         items * (steps + kSpanLead) < (1ll << 30) - pool->num_sms;
}

static bool shared_rows(const gc_kv_pool* pool, int32_t batch, int32_t max_shared_blocks,
                        int32_t max_blocks) {
  const int64_t blocks = static_cast<int64_t>(max_shared_blocks) + max_blocks;
  return row_by_row(pool, batch, blocks * pool->cfg.page_size, true);
}

// A shared call's workspace: the prefixes' pieces, the own parts, then the decode
// kernel's.
struct SharedSpace {
  SpanSpace span;
  size_t ml, o, decode, end;
};
static SharedSpace shared_space(const gc_kv_pool* pool, int32_t batch, int32_t groups,
                                int32_t max_shared_blocks, int32_t max_blocks,
                                int32_t num_q_heads) {
  SharedSpace s{};
  if (shared_rows(pool, batch, max_shared_blocks, max_blocks)) {
    s.end = decode_share_workspace_bytes(pool, num_q_heads);
    return s;
  }
  s.span = span_space(pool, batch, groups, max_shared_blocks, num_q_heads, true);
  const size_t rows = static_cast<size_t>(batch) * num_q_heads;
  s.ml = s.span.end;
  s.o = s.ml + (rows * sizeof(float2) + 255) / 256 * 256;
  s.decode = s.o + rows * pool->cfg.head_dim * sizeof(float);  // (rows of 256 bytes or more)
  const size_t shares = decode_share_workspace_bytes(pool, num_q_heads);  // (in the span kernel)
  const size_t alone = decode_workspace_bytes(pool, batch, max_blocks, num_q_heads);
  s.end = s.decode + (shares > alone ? shares : alone);
  return s;
}

size_t shared_decode_workspace_bytes(const gc_kv_pool* pool, int32_t batch, int32_t groups,
                                     int32_t max_shared_blocks, int32_t max_blocks,
                                     int32_t num_q_heads) {
  return shared_space(pool, batch, groups, max_shared_blocks, max_blocks, num_q_heads).end;
}

gc_status launch_shared_decode(const gc_kv_pool* pool, const SpanArgs& a, cudaStream_t stream) {
  const char* who = "gc_shared_prefix_decode_attn";
  const auto& cfg = pool->cfg;
  const SharedSpace space =
      shared_space(pool, a.batch, a.groups, a.max_shared_blocks, a.max_blocks, a.num_q_heads);
  gc_status st = check_space(who, space.end, a.workspace, a.workspace_bytes);
  if (st != GC_OK) return st;
  uint8_t* w = static_cast<uint8_t*>(a.workspace);
  if (shared_rows(pool, a.batch, a.max_shared_blocks, a.max_blocks))
    return launch_rows(pool, a, who, a.block_table, a.lens, a.max_blocks,
                       DecodePrefix{a.shared_table, a.shared_lens, a.start, nullptr, a.groups,
                                    a.max_shared_blocks}, stream);
  const SpanGeom span = span_geom(
      space.span, static_cast<int64_t>(a.max_shared_blocks) * cfg.page_size, true, w);
  DecodeArgs own{a.q, a.out, a.block_table, a.lens, a.batch, a.max_blocks, a.layer, a.num_q_heads,
                 a.softmax_scale, w + space.decode, space.end - space.decode, who,
                 DecodeParts{reinterpret_cast<float*>(w + space.o),
                             reinterpret_cast<float2*>(w + space.ml)}};
  const AttnArgs args{a.q, a.out, a.shared_table, a.shared_lens, nullptr, a.start, a.groups,
                      a.max_shared_blocks, a.layer, a.num_q_heads, a.batch, a.softmax_scale, who};
  if (decodes_in_kernel(pool, a)) {
    st = check_decode(pool, own);
    if (st != GC_OK) return st;
    const OwnDecode with{static_cast<const __nv_bfloat16*>(a.q), a.block_table, a.lens,
                         static_cast<float*>(own.workspace), pool->merge_counters,
                         decode_geom(pool, own, nullptr, nullptr), cfg.head_dim == 128 ? 15 : 5,
                         cfg.head_dim == 128 ? 4 : 1};
    st = launch_items(pool, args, span, stream, &with);
  } else {
    st = launch_decode(pool, own, stream);
    if (st == GC_OK) st = launch_items(pool, args, span, stream);
  }
  if (st != GC_OK) return st;
  const int64_t rows = static_cast<int64_t>(a.batch) * a.num_q_heads;
  const int per_block = 256 / (cfg.head_dim / 4);
  const auto join = cfg.head_dim == 128 ? shared_join_kernel<128> : shared_join_kernel<64>;
  return launch_join(pool, who, join, (rows + per_block - 1) / per_block, stream, span, a.lens,
                     static_cast<int>(static_cast<int64_t>(a.max_blocks) * cfg.page_size), own.own,
                     static_cast<__nv_bfloat16*>(a.out), a.num_q_heads,
                     a.num_q_heads / cfg.num_kv_heads, rows, pool->status, pool->span_counter);
}

}  // namespace gc

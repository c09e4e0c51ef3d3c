// Attention in which every row sees all keys of one or two page lists: cross
// attention (a request's new tokens over its cached states of another sequence)
// and decode behind a shared prefix (a request's one new token over its group's
// shared pages, then its own).  One warp per (row, q head), fp32 throughout,
// running maximum and sum over the keys read through the block tables.
#include "gc_internal.cuh"
#include "sm103_ptx.cuh"

namespace gc {
namespace {

using ptx::ex2_approx;

struct SpanGeom {
  int32_t Hq, Hkv, G, ps_shift, num_pages, layer, rows;
  int32_t count[2], width[2];  // table rows and columns: [0] requests, [1] groups
  float scale_log2;
};

template <int D>
struct RowState {
  static constexpr int E = D / 32;  // columns per lane
  float q[E], o[E], m, l;
};

// Keys [0, n) of table row `row`.  False if a page is bad (its keys are left out).
template <int D>
__device__ bool add_keys(RowState<D>& r, const uint8_t* pool, const int32_t* table, int64_t row,
                         int width, int n, int g, const SpanGeom& geo) {
  constexpr int E = RowState<D>::E;
  const int lane = threadIdx.x & 31, ps = 1 << geo.ps_shift;
  const int64_t plane = static_cast<int64_t>(geo.num_pages) * geo.Hkv * ps * D;
  const __nv_bfloat16* k =
      reinterpret_cast<const __nv_bfloat16*>(pool) + static_cast<int64_t>(geo.layer) * 2 * plane;
  bool good = true;
  for (int j = 0; j < n; ++j) {
    const int page = ld_plain(table + row * width + (j >> geo.ps_shift));
    if (page < 0 || page >= geo.num_pages) {
      good = false;
      continue;
    }
    const int64_t at = ((static_cast<int64_t>(page) * geo.Hkv + g) * ps + (j & (ps - 1))) * D + lane * E;
    float s = 0.f;
    for (int e = 0; e < E; ++e) s += r.q[e] * __bfloat162float(k[at + e]);
    for (int x = 16; x > 0; x >>= 1) s += __shfl_xor_sync(0xffffffffu, s, x);
    const float m = fmaxf(r.m, s);
    const float f = r.m == -INFINITY ? 0.f : ex2_approx(r.m - m), p = ex2_approx(s - m);
    r.m = m;
    r.l = r.l * f + p;
    for (int e = 0; e < E; ++e) r.o[e] = r.o[e] * f + p * __bfloat162float(k[plane + at + e]);
  }
  return good;
}

__device__ int last_start(const int32_t* start, int count, int t) {
  int lo = 0, hi = count;  // the last row whose start is <= t
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (ld_plain(start + mid) <= t) lo = mid; else hi = mid;
  }
  return lo;
}

// kShared: a row is a request, start[] the groups' first requests; otherwise a row
// is a new token, start[] the requests' first tokens.
template <int D, bool kShared>
__global__ void __launch_bounds__(128)
    span_attn_kernel(const __nv_bfloat16* q, const uint8_t* pool, const int32_t* table,
                     const int32_t* lens, const int32_t* shared_table, const int32_t* shared_lens,
                     const int32_t* start, __nv_bfloat16* out, SpanGeom geo, int32_t* status) {
  dependent_begin();
  constexpr int E = RowState<D>::E;
  const int lane = threadIdx.x & 31;
  const int64_t unit = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 5);
  if (unit >= static_cast<int64_t>(geo.rows) * geo.Hq) return;
  const int t = static_cast<int>(unit / geo.Hq), h = static_cast<int>(unit % geo.Hq);
  const int count = geo.count[kShared ? 1 : 0];
  const int s = last_start(start, count, t);
  const int begin = ld_plain(start + s), end = ld_plain(start + s + 1);
  bool good = begin >= 0 && t >= begin && t < end && end <= geo.rows;
  const int b = kShared ? t : s;
  const int n = good ? ld_plain(lens + b) : 0;
  const int S = good && kShared ? ld_plain(shared_lens + s) : 0;
  good = good && n >= 0 && S >= 0 && n <= static_cast<int64_t>(geo.width[0]) << geo.ps_shift &&
         (!kShared || S <= static_cast<int64_t>(geo.width[1]) << geo.ps_shift);
  if (good) {
    RowState<D> r;
    for (int e = 0; e < E; ++e) {
      r.q[e] = __bfloat162float(q[unit * D + lane * E + e]) * geo.scale_log2;
      r.o[e] = 0.f;
    }
    r.m = -INFINITY;
    r.l = 0.f;
    if (kShared) good = add_keys<D>(r, pool, shared_table, s, geo.width[1], S, h / geo.G, geo);
    good &= add_keys<D>(r, pool, table, b, geo.width[0], n, h / geo.G, geo);
    const float inv = r.l > 0.f ? 1.f / r.l : 0.f;  // no key: 0
    for (int e = 0; e < E; ++e) out[unit * D + lane * E + e] = __float2bfloat16_rn(r.o[e] * inv);
  }
  if (!good && lane == 0) record_error(status, GC_ERR_OUT_OF_RANGE);
}

template <bool kShared>
gc_status launch(const gc_kv_pool* pool, const SpanArgs& a, const char* who, cudaStream_t stream) {
  const auto& cfg = pool->cfg;
  SpanGeom geo;
  geo.Hq = a.num_q_heads;
  geo.Hkv = cfg.num_kv_heads;
  geo.G = geo.Hq / geo.Hkv;
  int s = 0;
  while ((1 << s) < cfg.page_size) ++s;
  geo.ps_shift = s;
  geo.num_pages = cfg.num_pages;
  geo.layer = a.layer;
  geo.rows = a.rows;
  geo.count[0] = a.batch;
  geo.count[1] = a.groups;
  geo.width[0] = a.max_blocks;
  geo.width[1] = a.max_shared_blocks;
  geo.scale_log2 = a.softmax_scale * 1.4426950408889634f;
  const int64_t grid = (static_cast<int64_t>(a.rows) * geo.Hq + 3) / 4;
  if (grid > 2147483647LL) return fail(GC_ERR_UNSUPPORTED, "%s: %d rows", who, a.rows);
  const auto kernel = cfg.head_dim == 128 ? span_attn_kernel<128, kShared> : span_attn_kernel<64, kShared>;
  const cudaError_t e = launch_dependent(
      kernel, static_cast<unsigned>(grid), 128, 0, stream, static_cast<const __nv_bfloat16*>(a.q),
      pool->data, a.block_table, a.lens, a.shared_table, a.shared_lens, a.start,
      static_cast<__nv_bfloat16*>(a.out), geo, pool->status);
  if (e != cudaSuccess) return cuda_fail(e, who);
  return GC_OK;
}

}  // namespace

gc_status launch_cross(const gc_kv_pool* pool, const SpanArgs& a, cudaStream_t stream) {
  return launch<false>(pool, a, "gc_paged_cross_attn", stream);
}

gc_status launch_shared_decode(const gc_kv_pool* pool, const SpanArgs& a, cudaStream_t stream) {
  return launch<true>(pool, a, "gc_shared_prefix_decode_attn", stream);
}

}  // namespace gc

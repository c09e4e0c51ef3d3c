// Whole pages between the 16-bit pool and the 4-bit cache (q4_format.cuh): packing pages
// that are finished, reading pages back, and reading back what one prefill call needs.
//
// All are element maps bound by HBM.  A warp takes eight rows at a time (pages have 16 or
// more, so they are of one page and head): four lanes a row read and write whole 64-byte
// pieces of the bf16 rows and the row's codes as one piece.
//
// Measured, 576 pages of 8 heads of 128 in 8 layers (302 MB in 16 bits, 85 in 4): packing 66
// us (5.8 TB/s), reading back 62 (6.2); what a prefill of 8 x (8192 + 1024) tokens reads (one
// layer, the same bytes) 61.
#include "q4_format.cuh"

namespace gc {
namespace {

constexpr int kThreads = 256;
constexpr int kWarpRows = 8;

struct PageGeom {
  Q4Geom q4;
  uint8_t* pool;  // bf16 pages [..][2][num_pages][Hkv][ps][d]
  int32_t num_pages, n, layer0, layers;
};

// Where the eight rows of a warp are in both forms, and the lane's row of them.
struct Rows {
  uint8_t *wide, *codes, *scales;
  bool ok;
};

// Part w of pages pool_ids[i] and q4_ids[i]: (i, layer, plane, head, eight rows).
template <int GR>
__device__ __forceinline__ Rows part_of(const PageGeom& g, uint64_t w, const int32_t* pool_ids,
                                        const int32_t* q4_ids, bool& is_k, int32_t* status) {
  const int parts = 1 << (g.q4.ps_shift - 3);
  const int slot = static_cast<int>(w & (parts - 1)) * kWarpRows + ((threadIdx.x & 31) >> 2);
  uint64_t rest = w >> (g.q4.ps_shift - 3);
  int h, kv, l;
  int64_t i;
  if (rest < 0xffffffffull) {  // (a 64-bit division is a call)
    uint32_t r = static_cast<uint32_t>(rest);
    h = static_cast<int>(r % g.q4.Hkv), r /= g.q4.Hkv;
    kv = static_cast<int>(r & 1), r >>= 1;
    l = static_cast<int>(r % g.layers);
    i = r / static_cast<uint32_t>(g.layers);
  } else {
    h = static_cast<int>(rest % g.q4.Hkv), rest /= g.q4.Hkv;
    kv = static_cast<int>(rest & 1), rest >>= 1;
    l = static_cast<int>(rest % g.layers);
    i = static_cast<int64_t>(rest / g.layers);
  }
  is_k = kv == 0;
  const int page = ld_plain(pool_ids + i), p4 = ld_plain(q4_ids + i);
  Rows r{nullptr, nullptr, nullptr, false};
  if (page < 0 || page >= g.num_pages || p4 < 0 || p4 >= g.q4.pages) {
    if ((w & (parts - 1)) == 0 && h == 0 && kv == 0 && l == 0 && (threadIdx.x & 31) == 0)
      record_error(status, GC_ERR_OUT_OF_RANGE);
    return r;
  }
  const uint64_t row =
      ((((static_cast<uint64_t>(l) + g.layer0) * 2 + kv) * g.num_pages + page) * g.q4.Hkv + h)
          << g.q4.ps_shift | slot;
  r.wide = g.pool + row * (64 * GR);
  uint8_t* head = q4_head(g.q4, l + g.layer0, kv, p4, h);
  r.codes = head + slot * (16 * GR);
  r.scales = head + (g.q4.ps * (16 * GR) + slot * (2 * GR));
  r.ok = true;
  return r;
}

template <int GR>
__global__ void __launch_bounds__(kThreads)
    pack_q4_kernel(const int32_t* pool_ids, const int32_t* q4_ids, PageGeom g, uint64_t parts,
                   int32_t* status) {
  dependent_begin();
  const uint64_t warps = static_cast<uint64_t>(gridDim.x) * (kThreads / 32);
  const int q = threadIdx.x & 3;
  for (uint64_t w = (static_cast<uint64_t>(blockIdx.x) * kThreads + threadIdx.x) >> 5; w < parts;
       w += warps) {
    bool is_k;
    const Rows r = part_of<GR>(g, w, pool_ids, q4_ids, is_k, status);
    if (!r.ok) continue;  // the whole warp
    uint4 x[GR];
#pragma unroll
    for (int i = 0; i < GR; ++i)
      x[i] = ld_plain(reinterpret_cast<const uint4*>(r.wide) + 4 * i + q);
    q4::store_row<GR>(x, is_k, r.codes, r.scales, true);
  }
}

template <int GR>
__global__ void __launch_bounds__(kThreads)
    unpack_q4_kernel(const int32_t* pool_ids, const int32_t* q4_ids, PageGeom g, uint64_t parts,
                     int32_t* status) {
  dependent_begin();
  const uint64_t warps = static_cast<uint64_t>(gridDim.x) * (kThreads / 32);
  const int q = threadIdx.x & 3;
  constexpr int U = 2;  // parts a warp has under way
  for (uint64_t w0 = (static_cast<uint64_t>(blockIdx.x) * kThreads + threadIdx.x) >> 5; w0 < parts;
       w0 += U * warps) {
    Rows r[U];
    bool is_k[U];
    uint32_t c[U][GR], s[U][GR / 2];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      r[u].ok = false;
      if (w0 + u * warps < parts)
        r[u] = part_of<GR>(g, w0 + u * warps, pool_ids, q4_ids, is_k[u], status);
      if (r[u].ok) q4::load_row<GR>(r[u].codes, r[u].scales, c[u], s[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (!r[u].ok) continue;
      uint4 x[GR];
      q4::expand_row<GR>(c[u], s[u], is_k[u], x);
#pragma unroll
      for (int i = 0; i < GR; ++i) reinterpret_cast<uint4*>(r[u].wide)[4 * i + q] = x[i];
    }
  }
}

// The 4-bit pages that one prefill call reads, one layer of them, as bf16 pages
// [2][to_pages][Hkv][ps][d].  A warp takes a plane's head of a page; the used positions of
// the tables are numbered request after request (a scan in every block), so that the
// work is dealt out evenly whatever the lengths.
template <int GR>
__global__ void __launch_bounds__(kThreads)
    unpack_q4_used_kernel(const int32_t* table, const int32_t* prefix_lens,
                          const int32_t* new_lens, PageGeom g, int32_t by_position,
                          int32_t batch, int32_t max_blocks) {
  extern __shared__ int start[];  // [batch + 1]
  __shared__ int scan[kThreads / 32];
  dependent_begin();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, q = lane & 3;
  int running = 0;
  for (int b0 = 0; b0 < batch; b0 += kThreads) {
    const int b = b0 + static_cast<int>(threadIdx.x);
    int pages = 0;
    if (b < batch) {
      const int P = ld_plain(prefix_lens + b), n = ld_plain(new_lens + b);
      if (n > 0 && P >= 0) {
        const int64_t T = static_cast<int64_t>(P) + n;
        pages = static_cast<int>(
            min(static_cast<int64_t>(max_blocks), (T + g.q4.ps - 1) >> g.q4.ps_shift));
      }
    }
    int incl = pages;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += y;
    }
    if (lane == 31) scan[warp] = incl;
    __syncthreads();
    int before = running;
#pragma unroll
    for (int i = 0; i < kThreads / 32; ++i) {
      if (i < warp) before += scan[i];
      running += scan[i];
    }
    if (b < batch) start[b] = before + incl - pages;
    __syncthreads();
  }
  if (threadIdx.x == 0) start[batch] = running;
  __syncthreads();
  const int64_t items = static_cast<int64_t>(running) * 2 * g.q4.Hkv;
  const int64_t warps = static_cast<int64_t>(gridDim.x) * (kThreads / 32);
  for (int64_t w = (static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x) >> 5; w < items;
       w += warps) {
    const int page = static_cast<int>(w / (2 * g.q4.Hkv));
    const int rest = static_cast<int>(w - static_cast<int64_t>(page) * 2 * g.q4.Hkv);
    const int kv = rest >= g.q4.Hkv, h = rest - kv * g.q4.Hkv;
    int lo = 0, hi = batch;  // the last request whose first page is <= page
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (start[mid] <= page) lo = mid; else hi = mid;
    }
    const int64_t at = static_cast<int64_t>(lo) * max_blocks + (page - start[lo]);
    const int p4 = ld_plain(table + at);
    if (p4 < 0 || p4 >= g.q4.pages) continue;  // the attention kernel reports the latter
    const uint8_t* head = q4_head(g.q4, g.layer0, kv, p4, h);
    const int64_t to = by_position ? at : p4;
    uint8_t* wide =
        g.pool + (((static_cast<uint64_t>(kv) * g.num_pages + to) * g.q4.Hkv + h) << g.q4.ps_shift) *
                     (64 * GR);
    for (int slot0 = lane >> 2; slot0 < g.q4.ps; slot0 += 2 * kWarpRows) {
      uint32_t c[2][GR], s[2][GR / 2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int slot = slot0 + u * kWarpRows;
        q4::load_row<GR>(head + slot * (16 * GR),
                         head + (g.q4.ps * (16 * GR) + slot * (2 * GR)), c[u], s[u]);
      }
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        uint4 x[GR];
        q4::expand_row<GR>(c[u], s[u], kv == 0, x);
        uint4* row = reinterpret_cast<uint4*>(wide + (slot0 + u * kWarpRows) * (64 * GR)) + q;
#pragma unroll
        for (int i = 0; i < GR; ++i) row[4 * i] = x[i];
      }
    }
  }
}

}  // namespace

gc_status launch_pages_q4(const gc_kv_pool* pool, const Q4Cache& cache, const int32_t* pool_ids,
                          const int32_t* q4_ids, int32_t n, int32_t layer0, int32_t layers,
                          bool pack, cudaStream_t stream) {
  const auto& cfg = pool->cfg;
  const PageGeom g{q4_geom(pool, cache), pool->data, cfg.num_pages, n, layer0, layers};
  const uint64_t parts = static_cast<uint64_t>(n) * layers * 2 * cfg.num_kv_heads *
                         (cfg.page_size / kWarpRows);
  uint64_t grid = (parts + kThreads / 32 - 1) / (kThreads / 32);
  const uint64_t cap = static_cast<uint64_t>(pool->num_sms) * 32;
  if (grid > cap) grid = cap;
  auto kernel = cfg.head_dim == 128 ? pack ? pack_q4_kernel<4> : unpack_q4_kernel<4>
                : pack              ? pack_q4_kernel<2>
                                    : unpack_q4_kernel<2>;
  const cudaError_t e = launch_dependent(kernel, static_cast<unsigned>(grid), kThreads, 0, stream,
                                         pool_ids, q4_ids, g, parts, pool->status);
  if (e != cudaSuccess)
    return cuda_fail(e, pack ? "gc_kv_pack_q4: kernel launch" : "gc_kv_unpack_q4: kernel launch");
  return GC_OK;
}

// Pages of scratch of a prefill call: one for each position of its tables, or for each page
// of the cache where those are fewer.
int64_t q4_scratch_pages(int32_t batch, int32_t max_blocks, int32_t q4_pages) {
  const int64_t positions = static_cast<int64_t>(batch) * max_blocks;
  return positions < q4_pages ? positions : q4_pages;
}

gc_status launch_prefill_q4(const gc_kv_pool* pool, const AttnArgs& a, const Q4Cache& cache,
                            void* workspace, cudaStream_t stream) {
  const auto& cfg = pool->cfg;
  gc_status st = check_item_bound(pool, a, pool->num_sms);
  if (st != GC_OK) return st;
  const int64_t pages = q4_scratch_pages(a.batch, a.max_blocks, cache.pages);
  const bool by_position = pages < cache.pages;
  // rows of the scratch are numbered with 32-bit ints, as the pool's are
  if (2ull * pages * cfg.num_kv_heads * cfg.page_size >= (1ull << 31))
    return fail(GC_ERR_UNSUPPORTED, "%s: %lld pages of scratch", a.who,
                static_cast<long long>(pages));
  const PageGeom g{q4_geom(pool, cache), static_cast<uint8_t*>(workspace),
                   static_cast<int32_t>(pages), 0, a.layer, 1};
  if (pages > 0) {
    const uint64_t items = static_cast<uint64_t>(a.batch) * a.max_blocks * 2 * cfg.num_kv_heads;
    uint64_t grid = (items + kThreads / 32 - 1) / (kThreads / 32);
    const uint64_t cap = static_cast<uint64_t>(pool->num_sms) * 8;
    if (grid > cap) grid = cap;
    const cudaError_t e = launch_dependent(
        cfg.head_dim == 128 ? unpack_q4_used_kernel<4> : unpack_q4_used_kernel<2>,
        static_cast<unsigned>(grid), kThreads, (static_cast<size_t>(a.batch) + 1) * sizeof(int),
        stream, cache.table, a.prefix_lens, a.new_lens, g, by_position ? 1 : 0, a.batch,
        a.max_blocks);
    if (e != cudaSuccess) return cuda_fail(e, a.who);
  }
  // (a cache without pages: nothing is read from there, but the maps want a tensor)
  const UnpackedPages u{static_cast<__nv_bfloat16*>(pages > 0 ? workspace : pool->data),
                        cache.table, static_cast<int32_t>(pages > 0 ? pages : 1), cache.pages,
                        by_position};
  return launch_attn_tc_unpacked(pool, a, u, stream);
}

}  // namespace gc

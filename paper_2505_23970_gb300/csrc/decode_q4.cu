// Paged decode attention over a cache in 4 bits (q4_format.cuh), one or a few tokens of
// every request: for request b with context length T, row i of its n last tokens, q head h
// and g = h / G,
//     out[b][i][h] = sum_{j < T - n + 1 + i} softmax_j(scale q[b][i][h] . k_j) v_j,
// k_j and v_j being c s of the codes and scales of the page (or a 16-bit page's values).
//
// Bound: HBM (9/32 of the bytes of 16-bit pages), with the instructions that a key takes
// close behind: the kernel has 3.5 times fewer cycles a key than the 16-bit one.  A warp's
// work on its keys is decode_q4.cuh's.
//
// Work split.  The keys of all (request, kv head) pairs are numbered in units of 32, a pair
// having kLead more of them for its fixed cost, and every warp has an equal share of the
// units, so that no warp waits for another before its share is done: a warp that comes to
// the end of a pair writes its rows and goes on with the next one.  (With a CTA's warps on
// one pair together, as in the 16-bit kernel, each change of pair cost it 5 us: 64 multi-turn
// contexts 103 us, by warps 79.)  Of a share, the first pair and the last may be parts of one;
// these are joined in fixed order, the parts of a CTA's warps through shared memory, those of
// several CTAs by the last of them to arrive (a counter per cut pair in the pool's control
// block).
//
// Measured (one call, back to back), 64/8 heads of 128 unless stated: 8 contexts of 9216
// keys (85 MB) 27 us; 64 multi-turn contexts, the newest page of each in 16 bits (307 MB) 68
// us; 8 of 65536 (604 MB) 115 us; 32 documents of up to 65536 (1.23 GB) 219-223 us, 5.5-5.6
// TB/s, 0.81-0.83 of the copy rate; 4 tokens each of 16 contexts of up to 8192, 32/8 heads
// (84 MB) 39 us; 8 of 65536 with heads of 64 (302 MB) 69 us, 4.4 TB/s.
// What holds it: copies of the kernel without its products | without its copies | whole, us:
// 8 of 65536 111 | 98 | 115, so the copies; the same with heads of 64 58 | 60 | 69 and 8 of
// 9216 17 | 22 | 26, neither alone; 16 columns over 94 MB 28 | 40 | 43, so the products.  No
// unit is full: in the first of these issue slots 59 %, ALU pipe (masks, shifts) 52 %, tensor
// pipe 38 %, DRAM 64 %.  Of the shorter calls 9 us are the start (look-ups, first loads: 4)
// and the joins (5).  With 16 columns a group takes 459 instead of 299 instructions and twice
// the products, by 8 warps an SM (12, with Q in shared memory to make room, took 41 us for 38).
// Spills: none with heads of 64 and 8 columns; with heads of 128 a few words outside the loop
// (7,000 of 78 million instructions); with heads of 64 and 16 columns in it, some 13 a pair of
// groups, 1.6 % of the instructions.
#include "decode_q4.cuh"

namespace gc {
namespace {

using dec::DecPiece;
using dec::Joined;
using dec::Keys4;

constexpr int kLead = 4;      // units without keys in front of each pair's
constexpr int kMinUnits = 2;  // of a warp's share, at least

// Warps of an SM, in one CTA, and stages of shared memory of a variant.  (Two CTAs of half
// the warps do not share the SM evenly: the one that came first is done with its equal
// share 15 % earlier, 8 contexts of 65536 keys 124 us for 119, both before the joins were
// what they are.)
template <int D, int NT>
struct Shape4 {
  static constexpr int kWarps = D * NT == 256 ? 8 : 16;
  static constexpr int kStages = 2;
  static constexpr int kThreads = 32 * kWarps;
  static constexpr int kHeads = 8 * NT;
  static constexpr int kStride = D + 4;                              // floats of a head
  static constexpr int kRingBytes = 2 * kStages * dec::Stage4<D>::kBytes;  // of a warp
  static constexpr int kPartBytes = kHeads * kStride * 4;
  static constexpr int kStaticBytes = kWarps * (1 + 32) * 4 + 16;  // the kernel's own arrays
  static_assert(kPartBytes <= kRingBytes, "a warp's last part lies over its stages");
};

// What a warp's part is of: a pair (request, kv head; -1: no part), and the CTAs with keys of
// the pair.
struct Part {
  int b, g, c0, c1;
};

// Shared memory: the warps' stages, over which the warps' last parts are kept, maxima and
// sums of their first and last parts, what these are of, the requests' first units and
// lengths, and the warps' first parts, as long as the batch leaves room for these (they are
// in the workspace else).
constexpr int kMostWithParts = 1024;  // requests
template <typename S>
constexpr size_t smem_bytes(int batch) {
  return S::kWarps * (S::kRingBytes + 2 * S::kHeads * sizeof(float2) + 2 * sizeof(Part) +
                      (batch <= kMostWithParts ? S::kPartBytes : 0)) +
         (2 * static_cast<size_t>(batch) + 4) / 4 * 4 * sizeof(int);
}
template <typename S>
constexpr size_t most_smem_bytes() {
  constexpr size_t few = smem_bytes<S>(kMostWithParts), many = smem_bytes<S>(kMaxBatch);
  return few > many ? few : many;
}

// Workspace: the CTAs' parts (O, then maxima and sums; two to a CTA), then the warps' first
// parts.
template <typename S, int D>
size_t workspace_bytes(int ctas, int batch) {
  return ctas * (2 * S::kHeads * (D + 2) * sizeof(float) +
                 (batch <= kMostWithParts ? 0 : S::kWarps * S::kPartBytes));
}

template <int D, int NT>
__global__ void __launch_bounds__(Shape4<D, NT>::kThreads, 1)
    decode_q4_kernel(const __nv_bfloat16* q, const int32_t* seq_lens, __nv_bfloat16* out,
                     float* ws, Dec4Geom geo, int32_t* status, int* merge_counters) {
  using S = Shape4<D, NT>;
  extern __shared__ __align__(16) uint8_t smem[];
  float2* mls = reinterpret_cast<float2*>(smem + S::kWarps * S::kRingBytes);
  Part* parts = reinterpret_cast<Part*>(mls + 2 * S::kWarps * S::kHeads);  // [warps][2]
  int* start = reinterpret_cast<int*>(parts + 2 * S::kWarps);              // [batch + 1]
  int* lens = start + geo.batch + 1;                                       // [batch]
  float2* ws_ml =
      reinterpret_cast<float2*>(ws + static_cast<int64_t>(gridDim.x) * 2 * S::kHeads * D);
  float* first_parts =
      geo.batch <= kMostWithParts
          ? reinterpret_cast<float*>(start + (2 * geo.batch + 4) / 4 * 4)
          : reinterpret_cast<float*>(ws_ml + static_cast<int64_t>(gridDim.x) * 2 * S::kHeads) +
                static_cast<int64_t>(blockIdx.x) * S::kWarps * S::kHeads * S::kStride;
  __shared__ int scan[S::kWarps], merge_flag[2], leaders_of[S::kWarps][32];
  static_assert(sizeof(scan) + sizeof(merge_flag) + sizeof(leaders_of) <= S::kStaticBytes, "room");
  dependent_begin();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int cta = blockIdx.x, warps = static_cast<int>(gridDim.x) * S::kWarps;

  // the units of each request, exclusive scan; a length outside [tokens, block table
  // capacity] is recorded
  {
    const int64_t cap = static_cast<int64_t>(geo.max_blocks) << geo.ps_shift;
    int running = 0;
    for (int b0 = 0; b0 < geo.batch; b0 += S::kThreads) {
      const int b = b0 + tid;
      int units = 0;
      if (b < geo.batch) {
        const int T = ld_plain(seq_lens + b);
        if (T >= geo.tokens && T <= cap)
          units = geo.Hkv * (kLead + ((T - 1) >> geo.unit_shift) + 1);
        else if (cta == 0)
          record_error(status, GC_ERR_OUT_OF_RANGE);
        lens[b] = T;
      }
      int incl = units;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += y;
      }
      if (lane == 31) scan[warp] = incl;
      __syncthreads();
      int before = running;
#pragma unroll
      for (int i = 0; i < S::kWarps; ++i) {
        if (i < warp) before += scan[i];
        running += scan[i];
      }
      if (b < geo.batch) start[b] = before + incl - units;
      __syncthreads();
    }
    if (tid == 0) start[geo.batch] = running;
    if (tid < 2 * S::kWarps) parts[tid].b = -1;
    __syncthreads();
  }
  const int total = start[geo.batch];
  const int per = max(kMinUnits, (total + warps - 1) / warps);
  const int cols = geo.G * geo.tokens;
  // a pair's first output (and q) row, and a column's row from there
  auto first_row = [&](int b, int g) {
    return static_cast<int64_t>(b) * geo.tokens * geo.Hq + g * geo.G;
  };
  auto row = [&](int h) { return (h >> geo.g_shift) * geo.Hq + (h & (geo.G - 1)); };

  // ---- this warp's units
  const int mine = cta * S::kWarps + warp;
  auto unit_of = [&](long long w) { return static_cast<int>(min(w * per, (long long)total)); };
  const int end = unit_of(mine + 1);
  for (int u = unit_of(mine); u < end;) {
    DecPiece w;
    w.b = dec::find_request(start, geo.batch, u);
    const int T = lens[w.b];
    const int local = u - start[w.b], nu = (start[w.b + 1] - start[w.b]) / geo.Hkv;
    w.g = local / nu;
    // units of the pair, counted from its first one with keys
    const int j = local - w.g * nu, last = min(nu, j + (end - u));
    const int j0 = max(0, j - kLead), j1 = last - kLead, all = nu - kLead;
    u += last - j;
    if (j1 <= 0) break;  // the share ends in front of the pair's first key
    w.k0 = j0 << geo.unit_shift;
    w.k1 = j1 == all ? T : j1 << geo.unit_shift;
    w.part = j0 == 0 && j1 == all ? -1 : j0 > 0 ? 0 : 1;
    Keys4<D, NT> keys;
    keys.template run<S::kStages>(
        smem + warp * S::kRingBytes, geo, w, T, q + first_row(w.b, w.g) * D, status);
    if (w.part < 0) {
      keys.store(out + first_row(w.b, w.g) * D, cols, row);
      continue;
    }
    // (the last part of a share lies over the warp's stages, which every lane has read)
    __syncwarp();
    keys.template keep<S::kStride>(
        w.part ? reinterpret_cast<float*>(smem + warp * S::kRingBytes)
               : first_parts + warp * S::kHeads * S::kStride,
        mls + (2 * warp + w.part) * S::kHeads);
    if (lane == 0) {
      const int pair0 = start[w.b] + w.g * nu;
      parts[2 * warp + w.part] = Part{w.b, w.g, (pair0 + kLead) / (per * S::kWarps),
                                      (pair0 + nu - 1) / (per * S::kWarps)};
    }
  }
  __syncthreads();

  // ---- the parts of this CTA's warps joined, pair by pair
  // Lane s has part s; those of a pair have the same key, and the first of them speaks for
  // the pair.  A pair with keys in other CTAs too leaves a part in the workspace, in the
  // CTA's first place if it began before the CTA, else in its second.
  static_assert(2 * S::kWarps <= 32, "a lane for every part");
  constexpr uint32_t kAll = 0xffffffffu;
  Part of{-1, 0, 0, 0};
  if (lane < 2 * S::kWarps) of = parts[lane];
  const uint32_t same =
      __match_any_sync(kAll, of.b < 0 ? -1 - lane : of.b * geo.Hkv + of.g);
  const bool leads = of.b >= 0 && (same & ((1u << lane) - 1)) == 0;
  const uint32_t leaders = __ballot_sync(kAll, leads);
  const int pairs = __popc(leaders);
  int* leader = leaders_of[warp];
  if (leads) leader[__popc(leaders & ((1u << lane) - 1))] = lane;
  __syncwarp();
  const uint32_t cut_bits[2] = {
      __ballot_sync(kAll, leads && of.c0 < cta),                   // (one lane at most)
      __ballot_sync(kAll, leads && of.c0 >= cta && of.c1 > cta)};  // (as well)
  const int quads = cols * (D / 4);  // four columns of a head each
  for (int i0 = 0; i0 < pairs * quads; i0 += S::kThreads) {
    const int i = i0 + tid, r = i / quads, x = i - r * quads;
    // (whole warps: the parts of a pair are another lane's to tell)
    const int s0 = r < pairs ? leader[r] : 0;
    uint32_t left = __shfl_sync(kAll, same, s0);
    if (r >= pairs) continue;
    const int h = x / (D / 4), d = 4 * (x % (D / 4));
    Joined sum;
    while (left) {
      float2 ml[4];
      float4 o[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int s = left ? __ffs(left) - 1 : s0;
        const float* from = s & 1
                                ? reinterpret_cast<const float*>(smem + (s >> 1) * S::kRingBytes)
                                : first_parts + (s >> 1) * S::kHeads * S::kStride;
        ml[k] = left ? mls[s * S::kHeads + h] : make_float2(dec::kNone, 0.f);
        o[k] = left ? *reinterpret_cast<const float4*>(from + h * S::kStride + d)
                    : make_float4(0.f, 0.f, 0.f, 0.f);
        left &= left - 1;
      }
      sum.add(ml, o);
    }
    if (((cut_bits[0] | cut_bits[1]) >> s0 & 1) == 0) {
      sum.store(out + (first_row(parts[s0].b, parts[s0].g) + row(h)) * D + d);
    } else {
      const int64_t at = (static_cast<int64_t>(cta) * 2 + (cut_bits[1] >> s0 & 1)) * S::kHeads + h;
      *reinterpret_cast<float4*>(ws + at * D + d) = sum.o;
      if (d == 0) ws_ml[at] = make_float2(sum.M, sum.L);
    }
  }
  // ---- the last CTA with keys of a cut pair joins the CTAs' parts
  if ((cut_bits[0] | cut_bits[1]) == 0) return;  // (the same in every thread)
  __syncthreads();
  // (the barrier has the CTA's parts before the fence of the one thread that counts)
  if (tid < 2) {
    int last = 0;
    if (const uint32_t bits = tid ? cut_bits[1] : cut_bits[0]) {
      const Part cut = parts[__ffs(bits) - 1];
      __threadfence();
      last = atomicAdd(merge_counters + cut.c0, 1) == cut.c1 - cut.c0;
      if (last) merge_counters[cut.c0] = 0;
      __threadfence();
    }
    merge_flag[tid] = last;
  }
  __syncthreads();
  for (int i = tid; i < 2 * quads; i += S::kThreads) {
    const int k0 = i >= quads, x = i - k0 * quads;
    if (!merge_flag[k0]) continue;
    const Part cut = parts[__ffs(k0 ? cut_bits[1] : cut_bits[0]) - 1];
    const int h = x / (D / 4), d = 4 * (x % (D / 4));
    Joined sum;
    for (int c = cut.c0; c <= cut.c1; c += 8) {
      float2 ml[8];
      float4 o[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int64_t at = (static_cast<int64_t>(c + k) * 2 + (c + k == cut.c0)) * S::kHeads + h;
        ml[k] = c + k <= cut.c1 ? __ldcg(ws_ml + at) : make_float2(dec::kNone, 0.f);
        o[k] = c + k <= cut.c1 ? __ldcg(reinterpret_cast<const float4*>(ws + at * D + d))
                               : make_float4(0.f, 0.f, 0.f, 0.f);
      }
      sum.add(ml, o);
    }
    sum.store(out + (first_row(cut.b, cut.g) + row(h)) * D + d);
  }
}

template <int D, int NT>
gc_status launch(const gc_kv_pool* pool, const DecodeArgs& a, const Dec4Geom& geo,
                 cudaStream_t stream) {
  using S = Shape4<D, NT>;
  const int grid = min(pool->num_sms, kMergeCounters);
  const size_t need = workspace_bytes<S, D>(grid, a.batch);
  if (a.workspace == nullptr || a.workspace_bytes < need)
    return fail(GC_ERR_INVALID_ARG,
                "%s: workspace of %zu bytes needed (gc_paged_decode_q4_workspace_bytes), got %zu",
                a.who, need, a.workspace_bytes);
  const size_t smem = smem_bytes<S>(a.batch);
  auto kernel = decode_q4_kernel<D, NT>;
  static_assert(most_smem_bytes<S>() + S::kStaticBytes <= 227 * 1024, "room");
  cudaError_t e = allow_shared<most_smem_bytes<S>()>(kernel);
  if (e != cudaSuccess) return cuda_fail(e, a.who);
  e = launch_dependent(kernel, grid, S::kThreads, smem, stream,
                       static_cast<const __nv_bfloat16*>(a.q), a.seq_lens,
                       static_cast<__nv_bfloat16*>(a.out), static_cast<float*>(a.workspace), geo,
                       pool->status, pool->merge_counters);
  if (e != cudaSuccess) return cuda_fail(e, a.who);
  return GC_OK;
}

int ilog2(int x) {
  int s = 0;
  while ((1 << s) < x) ++s;
  return s;
}

}  // namespace

size_t decode_q4_workspace_bytes(const gc_kv_pool* pool, int32_t batch, int32_t num_q_heads,
                                 int32_t tokens) {
  const int ctas = min(pool->num_sms, kMergeCounters);
  const bool narrow = num_q_heads / pool->cfg.num_kv_heads * tokens <= 8;
  if (pool->cfg.head_dim == 128)
    return narrow ? workspace_bytes<Shape4<128, 1>, 128>(ctas, batch)
                  : workspace_bytes<Shape4<128, 2>, 128>(ctas, batch);
  return narrow ? workspace_bytes<Shape4<64, 1>, 64>(ctas, batch)
                : workspace_bytes<Shape4<64, 2>, 64>(ctas, batch);
}

gc_status launch_decode_q4(const gc_kv_pool* pool, const DecodeArgs& a, const Q4Cache& cache,
                           int32_t tokens, cudaStream_t stream) {
  const auto& cfg = pool->cfg;
  gc_status st = check_decode(pool, a);
  if (st != GC_OK) return st;
  Dec4Geom geo;
  geo.batch = a.batch;
  geo.Hq = a.num_q_heads;
  geo.Hkv = cfg.num_kv_heads;
  geo.G = geo.Hq / geo.Hkv;
  geo.g_shift = ilog2(geo.G);
  geo.tokens = tokens;
  geo.ps = cfg.page_size;
  geo.ps_shift = ilog2(cfg.page_size);
  geo.num_pages = cfg.num_pages;
  geo.q4_pages = cache.pages;
  geo.max_blocks = a.max_blocks;
  geo.scale_log2 = a.softmax_scale * 1.4426950408889634f;
  const uint64_t head = q4_head_bytes(cfg.head_dim, cfg.page_size);
  geo.q4_page = static_cast<uint32_t>(geo.Hkv * head);
  geo.q4_plane = static_cast<int64_t>(cache.pages) * geo.q4_page;
  geo.plane16 = static_cast<int64_t>(cfg.num_pages * page_bytes(cfg));
  geo.q4_k = cache.data + 2 * a.layer * geo.q4_plane;
  geo.pool_k = pool->data + 2 * a.layer * geo.plane16;
  geo.q4_table = cache.table;
  geo.block_table = a.block_table;
  if (geo.Hkv * head > UINT32_MAX)
    return fail(GC_ERR_UNSUPPORTED, "%s: pages of %llu bytes", a.who,
                static_cast<unsigned long long>(geo.Hkv * head));
  // units are numbered with 32-bit ints, with a margin for the shares' rounding
  const int64_t cap = static_cast<int64_t>(a.max_blocks) * cfg.page_size;
  const int64_t pairs = static_cast<int64_t>(a.batch) * geo.Hkv;
  const int64_t margin = 1 << 16;
  geo.unit_shift = 5;
  while (geo.unit_shift < 12 &&
         pairs * (((cap - 1) >> geo.unit_shift) + 1 + kLead) > INT32_MAX - margin)
    ++geo.unit_shift;
  if (pairs * (((cap - 1) >> geo.unit_shift) + 1 + kLead) > INT32_MAX - margin)
    return fail(GC_ERR_UNSUPPORTED, "%s: %lld pairs of up to %lld keys", a.who,
                static_cast<long long>(pairs), static_cast<long long>(cap));
  const bool narrow = geo.G * tokens <= 8;
  if (cfg.head_dim == 128)
    return narrow ? launch<128, 1>(pool, a, geo, stream) : launch<128, 2>(pool, a, geo, stream);
  return narrow ? launch<64, 1>(pool, a, geo, stream) : launch<64, 2>(pool, a, geo, stream);
}

}  // namespace gc

// Attention whose rows see all keys of a request (cross attention) or of a group's
// shared prefix, on the tensor-core kernels: how a call's work is dealt out, and where
// the pieces' results go until they are joined.
//
// An item is a kv head and 256 q rows of a request (or group), over all of its keys in
// steps of 128.  Two ways:
//  * whole items, handed out one by one;
//  * equal shares: all items' steps, each item with an allowance for its fixed cost in
//    front, numbered in order (units) and cut into one contiguous share per worker, so
//    that every SM is busy for the same time however few the items are and however
//    their lengths differ.  An item that a share boundary cuts is done in pieces, whose
//    results (the rows' O, unscaled, reference maximum in log2 units and sum, in
//    binary32) are joined afterwards:
//        out = sum_s O_s 2^(m_s - M) / sum_s l_s 2^(m_s - M),  M = max_s m_s.
//    A share has at most two such pieces: its first (slot 0), and its last (slot 1).
#pragma once

#include "decode_mma.cuh"
#include "gc_internal.cuh"
#include "sm103_ptx.cuh"

namespace gc {

// The own keys of the requests behind shared prefixes, decoded by some of the CTAs of the
// kernel that works on the prefixes: alone, each of the two leaves SMs idle at its start
// and end, and the first is bound by latencies where the second is bound by memory.
struct OwnDecode {
  const __nv_bfloat16* q;
  const int32_t* block_table;
  const int32_t* lens;
  float* workspace;
  int* merge_counters;
  DecGeom geo;
  int32_t weight;  // time of 128 own keys and a kv head on one SM, in eighths of a unit
};

constexpr int kSpanRows = 256;      // q rows of an item
constexpr int kSpanRequests = 512;  // most requests of a call that is cut into shares
// An item costs about this many steps beyond its own (its first scores, the last
// product and the results), a join about kSpanJoin.
constexpr int kSpanLead = 2;
constexpr int kSpanJoin = 4;
constexpr int kSpanMinShare = 4;

struct SpanGeom {
  int32_t cap;      // keys a block-table row can hold
  int32_t workers;  // CTAs (pairs) that take items
  int32_t stride;   // rows of a slot
  int32_t cuts;     // items may be cut
  int32_t shared;   // requests are groups (new_lens is not given); whole items' results
                    // go to `whole`, not to the output
  int32_t* plan;    // SpanPlan, for the joins
  int4* prior;      // shared: per request, see SpanPrior
  DecodeParts whole;  // shared: [request][q head]
  float2* ml;       // [2 * workers][stride]: reference maximum, sum
  float* o;         // [2 * workers][stride][d]
};

// The plan in the workspace: [0] units of a share, 0: whole items; [1] all units;
// where items may be cut: [2] requests, then from kPlanStart each one's first unit (and
// the end), from kPlanOrder its number.
constexpr int kPlanStart = 4, kPlanOrder = kPlanStart + kSpanRequests + 4;
constexpr int kPlanWords = kPlanOrder + kSpanRequests;

// A request of a shared prefix, as an int4: its G rows of kv head g are rows
// [row, row + G) of the item whose first unit is unit + g * head_units.  steps: of the
// item; 0: no shared keys, -1: the request is skipped.
struct SpanPrior {
  int32_t unit, head_units, steps, row;
};

// One request's rows, keys and first token; rows 0 if there is nothing to do.
struct SpanRequest {
  int n, T, cu;
  bool bad;
};
__device__ __forceinline__ SpanRequest span_request(const SpanGeom& sp, int b, int total_new,
                                                    const int32_t* lens, const int32_t* new_lens,
                                                    const int32_t* cu) {
  SpanRequest r;
  r.T = ld_plain(lens + b);
  r.cu = ld_plain(cu + b);
  const int64_t n = sp.shared ? static_cast<int64_t>(ld_plain(cu + b + 1)) - r.cu
                              : ld_plain(new_lens + b);
  r.bad = n < 0 || r.cu < 0 || r.cu + n > total_new || (n > 0 && (r.T < 0 || r.T > sp.cap));
  r.n = r.bad ? 0 : static_cast<int>(n);
  return r;
}
__device__ __forceinline__ int span_steps(int T) { return T > 0 ? ((T - 1) >> 7) + 1 : 0; }
__device__ __forceinline__ int span_tiles(int n, int G) {
  return (n * G + kSpanRows - 1) / kSpanRows;
}

// Units of a share, 0 for whole items, and the workers that take part, worked out by one
// warp; every CTA comes to the same answer.  request(b) gives a SpanRequest.
// own: the other workers decode own keys (shares always; own->geo.batch requests).
constexpr int kSpanStart = 9;  // units in the time that a span CTA takes beyond an own one's
struct SpanPlan {
  int share, workers;
};
template <typename F>
__device__ SpanPlan span_plan(const SpanGeom& sp, int batch, int Hkv, int G, const OwnDecode* own,
                              int sms_per_worker, F request) {
  if (!sp.cuts || batch > kSpanRequests) return {0, sp.workers};
  const int lane = threadIdx.x & 31;
  long long units = 0, items = 0;
  int most = 0;
  for (int b = lane; b < batch; b += 32) {
    const SpanRequest r = request(b);
    const int st = r.n > 0 ? span_steps(r.T) : 0;
    if (st == 0) continue;
    const long long n = static_cast<long long>(Hkv) * span_tiles(r.n, G);
    items += n;
    units += n * (st + kSpanLead);
    most = max(most, st + kSpanLead);
  }
  long long keys = 0;  // own ones, a pair's fixed cost counted as 128
  if (own)
    for (int b = lane; b < own->geo.batch; b += 32) {
      const int T = ld_plain(own->lens + b);
      if (T > 0) keys += T + 128ll;
    }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    units += __shfl_xor_sync(0xffffffffu, units, o);
    items += __shfl_xor_sync(0xffffffffu, items, o);
    if (own) keys += __shfl_xor_sync(0xffffffffu, keys, o);
  }
  most = __reduce_max_sync(0xffffffffu, most);
  if (own) {
    // the number of span workers for which the slower side is fastest
    if (units == 0) return {kSpanMinShare, 0};
    const float u = static_cast<float>(units);
    const float o = static_cast<float>(keys) * Hkv * own->weight * (1.f / (128 * 8));
    float best = INFINITY;
    int n = 1;
    for (int w = 1 + lane; w < sp.workers; w += 32) {
      const float t = fmaxf(fmaxf(u / w, kSpanMinShare) + kSpanStart,
                            o / ((sp.workers - w) * sms_per_worker));
      if (t < best) best = t, n = w;
    }
    const unsigned t = __reduce_min_sync(0xffffffffu, __float_as_uint(best));  // (positive)
    n = __reduce_min_sync(0xffffffffu, __float_as_uint(best) == t ? n : sp.workers);
    return {max(static_cast<int>((units + n - 1) / n), kSpanMinShare), n};
  }
  if (units + sp.workers >= (1ll << 30)) return {0, sp.workers};  // units are 32-bit ints
  // Time in steps: of whole items, in rounds of the longest or as the last of them ends,
  // against equal shares and their join.
  const long long even = (units + sp.workers - 1) / sp.workers;
  const long long rounds = (items + sp.workers - 1) / sp.workers;
  const long long whole = min(rounds * most, even + most);
  const long long share = max(even, static_cast<long long>(kSpanMinShare));
  return {share + kSpanJoin < whole ? static_cast<int>(share) : 0, sp.workers};
}

// The place of a request's items in work order; start: first unit (shares) or item.
__device__ __forceinline__ int span_place(const int* start, int batch, int u) {
  int lo = 0, hi = batch;  // the last place whose start is <= u
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (start[mid] <= u) lo = mid; else hi = mid;
  }
  return lo;
}

// The work at unit u of a share that ends before unit `end` (shares), or at item u
// (share 0).  nt 0: there is none left in the share.  slot: of its pieces, -1 if it is a
// whole item; next: the unit after it.
struct SpanPiece {
  int b, g, tile, n, T, cu, j0, nt, slot, next;
};
template <typename F>
__device__ __forceinline__ SpanPiece span_piece(int u, int share, int worker, int end, int batch,
                                                const int* start, const int16_t* order, int Hkv,
                                                int G, F request) {
  SpanPiece w;
  const int p = span_place(start, batch, u);
  w.b = batch <= kSpanRequests ? order[p] : p;
  const SpanRequest r = request(w.b);
  w.n = r.n;
  w.T = r.T;
  w.cu = r.cu;
  const int steps = span_steps(r.T), tiles = span_tiles(r.n, G), local = u - start[p];
  int item = local;
  w.j0 = 0;
  w.nt = steps;
  w.slot = -1;
  w.next = u + 1;
  if (share) {
    const int per = steps + kSpanLead;
    item = local / per;
    const int off = local - item * per, to = min(per, off + (end - u));
    w.j0 = max(0, off - kSpanLead);
    w.nt = max(0, to - kSpanLead - w.j0);
    if (w.nt < steps) w.slot = 2 * worker + (u == worker * share ? 0 : 1);
    w.next = u + to - off;
  }
  // the tiles that read the same keys one after the other
  w.g = item / tiles;
  w.tile = item - w.g * tiles;
  return w;
}

// Pieces of the item whose first unit is u0: of shares c0 to c1, the first in slot
// `first` of c0's, the others in slot 0.
struct SpanCut {
  int c0, c1, first;
};
__device__ __forceinline__ SpanCut span_cut(int u0, int steps, int share) {
  SpanCut c;
  c.c0 = (u0 + kSpanLead) / share;
  c.c1 = (u0 + kSpanLead + steps - 1) / share;
  c.first = c.c0 * share >= u0 ? 0 : 1;
  return c;
}

// Thread `me` of `all`: the plan for the joins, where items may be cut.
__device__ inline void span_write_plan(const SpanGeom& sp, int batch, int share, const int* start,
                                       const int16_t* order, int64_t me, int64_t all) {
  if (!sp.plan) return;
  if (me == 0) {
    sp.plan[0] = share;
    sp.plan[1] = start[batch];
    sp.plan[2] = batch;
  }
  if (share == 0 || sp.shared) return;
  for (int64_t p = me; p <= batch; p += all) {
    sp.plan[kPlanStart + p] = start[p];
    if (p < batch) sp.plan[kPlanOrder + p] = order[p];
  }
}

// Thread `me` of `all`: the requests' rows of the groups' items.  first_of: each
// group's first unit or item.
__device__ inline void span_priors(const SpanGeom& sp, int groups, int G, int batch,
                                   const int* first_of, const int32_t* lens, const int32_t* cu,
                                   int64_t me, int64_t all) {
  for (int64_t b = me; b < batch; b += all) {
    int lo = 0, hi = groups;  // the last group whose first request is <= b
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (ld_plain(cu + mid) <= b) lo = mid; else hi = mid;
    }
    const SpanRequest r = span_request(sp, lo, batch, lens, nullptr, cu);
    SpanPrior p{0, 0, -1, 0};
    if (!r.bad && b >= r.cu && b < r.cu + r.n) {
      const int row = (static_cast<int>(b) - r.cu) * G, per = span_steps(r.T) + kSpanLead;
      p.steps = span_steps(r.T);
      p.unit = first_of[lo] + row / kSpanRows * per;
      p.head_units = span_tiles(r.n, G) * per;
      p.row = row % kSpanRows;
    }
    sp.prior[b] = make_int4(p.unit, p.head_units, p.steps, p.row);
  }
}

// Thread `me` of `all` (whole warps): zeros for the rows of requests without keys.
__device__ inline void span_zeros(const SpanGeom& sp, int batch, int Hq, int D, int total_new,
                                  const int32_t* lens, const int32_t* new_lens, const int32_t* cu,
                                  __nv_bfloat16* out, int64_t me, int64_t all) {
  const int lane = threadIdx.x & 31;
  for (int b0 = 0; b0 < batch; b0 += 32) {
    const bool none = b0 + lane < batch && ld_plain(lens + b0 + lane) == 0;
    uint32_t which = __ballot_sync(0xffffffffu, none);
    for (; which; which &= which - 1) {
      const SpanRequest r = span_request(sp, b0 + __ffs(which) - 1, total_new, lens, new_lens, cu);
      const int64_t words = static_cast<int64_t>(r.n) * Hq * D / 8;
      uint4* dst = reinterpret_cast<uint4*>(out) + static_cast<int64_t>(r.cu) * Hq * D / 8;
      for (int64_t i = me; i < words; i += all) dst[i] = make_uint4(0, 0, 0, 0);
    }
  }
}

// ------------------------------------------------------------------ host side
// A call's workspace: where its parts are, in bytes from its start.
struct SpanSpace {
  int64_t slots, stride;
  size_t plan, prior, whole_ml, whole_o, ml, o, end;
};
inline SpanSpace span_space(const gc_kv_pool* pool, int64_t rows, int64_t batch, int64_t max_blocks,
                            int num_q_heads, bool shared) {
  SpanSpace s{};
  const auto& c = pool->cfg;
  const int64_t G = num_q_heads / c.num_kv_heads;
  const int64_t steps = (max_blocks * c.page_size + 127) / 128;
  const int64_t workers = c.head_dim == 128 ? pool->num_sms / 2 : pool->num_sms;
  // (items of two steps are too short to be cut)
  s.slots = (shared || steps > 2) && batch <= kSpanRequests ? 2 * workers : 0;
  s.stride = rows * G < kSpanRows ? rows * G : kSpanRows;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t x = at;
    at += (bytes + 255) / 256 * 256;
    return x;
  };
  const size_t out_rows = static_cast<size_t>(rows) * num_q_heads, row = c.head_dim * sizeof(float);
  s.plan = take(shared || s.slots ? kPlanWords * sizeof(int32_t) : 0);
  s.prior = take(shared ? rows * sizeof(int4) : 0);
  s.whole_ml = take(shared ? out_rows * sizeof(float2) : 0);
  s.whole_o = take(shared ? out_rows * row : 0);
  s.ml = take(static_cast<size_t>(s.slots * s.stride) * sizeof(float2));
  s.o = take(static_cast<size_t>(s.slots * s.stride) * row);
  s.end = at;
  return s;
}

inline SpanGeom span_geom(const SpanSpace& s, int64_t cap, bool shared, void* workspace) {
  uint8_t* w = static_cast<uint8_t*>(workspace);
  SpanGeom g{};
  g.cap = static_cast<int32_t>(cap);
  g.stride = static_cast<int32_t>(s.stride);
  g.cuts = s.slots > 0;
  g.shared = shared ? 1 : 0;
  g.plan = shared || s.slots ? reinterpret_cast<int32_t*>(w + s.plan) : nullptr;
  g.prior = shared ? reinterpret_cast<int4*>(w + s.prior) : nullptr;
  if (shared)
    g.whole = DecodeParts{reinterpret_cast<float*>(w + s.whole_o),
                          reinterpret_cast<float2*>(w + s.whole_ml)};
  g.ml = reinterpret_cast<float2*>(w + s.ml);
  g.o = reinterpret_cast<float*>(w + s.o);
  return g;
}

}  // namespace gc

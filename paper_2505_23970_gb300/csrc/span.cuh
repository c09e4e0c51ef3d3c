// Attention whose rows see all keys of a request (cross attention) or of a group's
// shared prefix, on the tensor-core kernels: how a call's work is cut, and where the
// pieces' results go until they are joined.
//
// A request's (or group's) item is a kv head and 256 of its q rows, over all of its
// keys.  Where the items do not fill the GPU evenly, the keys of the long ones are
// cut into parts of `steps` 128-key steps; a part's result (a piece) is its rows' O,
// unscaled, reference maximum in log2 units and sum, in binary32:
//     out = sum_s O_s 2^(m_s - M) / sum_s l_s 2^(m_s - M),  M = max_s m_s.
#pragma once

#include "gc_internal.cuh"
#include "sm103_ptx.cuh"

namespace gc {

constexpr int kSpanRows = 256;       // q rows of an item
constexpr int kSpanWhole = 1 << 24;  // steps of a part that is never reached: no cuts
// Rounds of pieces over the workers that a plan may take.  More rounds even out the
// rest of the last one, but each piece costs about three steps beyond its own.
constexpr int kSpanRounds = 4;
constexpr int kSpanPieceSteps = 3;
constexpr int kSpanMinSteps = 2;

struct SpanGeom {
  int32_t cap;      // keys a block-table row can hold
  int32_t workers;  // CTAs (pairs) that take items
  int32_t pieces;   // pieces that the workspace holds
  int32_t stride;   // rows of a piece there
  int32_t shared;   // requests are groups (new_lens is not given) and every item writes a piece
  int4* prior;      // shared: per request, see SpanPrior
  int32_t* cut;     // otherwise: what the join needs to know, see SpanCut
  float2* ml;       // [pieces][stride] reference maximum, sum
  float* o;         // [pieces][stride][d]
};

// Per request of a shared prefix (an int4): its G rows of kv head g are rows
// [row, row + G) of pieces base + (g * parts + part) * tiles, part < parts.
// parts 0: no shared keys, -1: the request is skipped.
struct SpanPrior {
  int32_t base, tiles, parts, row;
};

// In front of the pieces of cut requests: [0] requests that are cut (they are the
// longest, so the first in work order, and piece = item), [1] steps of a part, then
// from kCutFirst each one's first item, and from kCutOrder its number.
constexpr int kCutRequests = 512;
constexpr int kCutFirst = 4, kCutOrder = kCutFirst + kCutRequests + 4;
constexpr int kCutWords = kCutOrder + kCutRequests;

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
__device__ __forceinline__ int span_parts(int steps, int part_steps) {
  return steps == 0 ? 0 : (steps - 1) / part_steps + 1;
}

// Steps of a part, worked out by one warp: of a few lengths around an equal share for
// each of 1 to kSpanRounds rounds, the one whose rounds take the least time.  Every
// CTA comes to the same answer.  request(b) gives a SpanRequest.
template <typename F>
__device__ int span_plan(const SpanGeom& sp, int batch, int Hkv, int G, bool may_cut, F request) {
  const int lane = threadIdx.x & 31;
  if (!may_cut) return kSpanWhole;
  long long total = 0;
  int most = 0;
  SpanRequest mine{0, 0, 0, false};
  for (int b = lane; b < batch; b += 32) {
    mine = request(b);
    if (mine.n == 0) mine.T = 0;
    const int st = span_steps(mine.T);
    total += static_cast<long long>(Hkv) * span_tiles(mine.n, G) * st;
    most = max(most, st);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
  most = __reduce_max_sync(0xffffffffu, most);
  constexpr int kSlacks = 4, kPlans = kSpanRounds * kSlacks;
  int steps[kPlans], items[kPlans], cut[kPlans];
#pragma unroll
  for (int p = 0; p < kPlans; ++p) {
    // an equal share, and 1/8, 2/8, 3/8 more: parts are rounded up to whole items
    const long long share = total * (8 + p % kSlacks) /
                            (8ll * (p / kSlacks + 1) * sp.workers) + 1;
    steps[p] = static_cast<int>(min(max(share, static_cast<long long>(kSpanMinSteps)),
                                    static_cast<long long>(kSpanWhole)));
    items[p] = cut[p] = 0;
  }
  for (int b0 = 0; b0 < batch; b0 += 32) {
    SpanRequest r = mine;
    if (batch > 32) {
      r = SpanRequest{0, 0, 0, false};
      if (b0 + lane < batch) r = request(b0 + lane);
    }
    const int st = r.n > 0 ? span_steps(r.T) : 0, one = Hkv * span_tiles(r.n, G);
#pragma unroll
    for (int p = 0; p < kPlans; ++p) {
      const int parts = span_parts(st, steps[p]);
      items[p] += one * parts;
      cut[p] += parts > 1 ? one * parts : 0;
    }
  }
  int best = kSpanWhole;
  long long cost = 0x7fffffffffffffffll;
#pragma unroll
  for (int p = 0; p < kPlans; ++p) {
    const int n = __reduce_add_sync(0xffffffffu, items[p]);
    const int c = __reduce_add_sync(0xffffffffu, cut[p]);
    const long long rounds = (n + sp.workers - 1) / sp.workers;
    const long long t = rounds * (min(steps[p], most) + kSpanPieceSteps);
    if ((sp.shared ? n : c) <= sp.pieces && t < cost) {
      cost = t;
      best = steps[p];
    }
  }
  return best;
}

// Thread `me` of `all`: the requests' rows of the groups' pieces.  first_of: each
// group's first item; none: no items are worked on.
__device__ inline void span_priors(const SpanGeom& sp, int groups, int G, int batch,
                                   int part_steps, bool none, const int* first_of,
                                   const int32_t* lens, const int32_t* cu, int64_t me,
                                   int64_t all) {
  for (int64_t b = me; b < batch; b += all) {
    int lo = 0, hi = groups;  // the last group whose first request is <= b
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (ld_plain(cu + mid) <= b) lo = mid; else hi = mid;
    }
    const SpanRequest r = span_request(sp, lo, batch, lens, nullptr, cu);
    SpanPrior p{0, 0, -1, 0};
    if (!r.bad && !none && b >= r.cu && b < r.cu + r.n) {
      const int row = (static_cast<int>(b) - r.cu) * G;
      p.tiles = span_tiles(r.n, G);
      p.parts = span_parts(span_steps(r.T), part_steps);
      p.base = first_of[lo] + row / kSpanRows;
      p.row = row % kSpanRows;
    }
    sp.prior[b] = make_int4(p.base, p.tiles, p.parts, p.row);
  }
}

// Thread `me` of `all` (whole warps): zeros for the rows of requests without keys, and
// what the join of cut requests needs to know.  (order: the requests in work order,
// where there are at most kCutRequests.)
__device__ inline void span_empty_and_cut(const SpanGeom& sp, int batch, int Hq, int D,
                                          int total_new, int part_steps, const int* item_start,
                                          const int16_t* order, const int32_t* lens,
                                          const int32_t* new_lens, const int32_t* cu,
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
  if (sp.pieces == 0) return;
  if (me == 0) sp.cut[1] = part_steps;
  if (batch > kCutRequests) {  // (not cut)
    if (me == 0) sp.cut[0] = 0;
    return;
  }
  // the cut ones are the longest; a bad one among them has no items
  auto is_cut = [&](int64_t p) {
    return p < batch && span_steps(ld_plain(lens + order[p])) > part_steps;
  };
  if (me == 0 && !is_cut(0)) sp.cut[0] = 0;
  for (int64_t p = me; p < batch; p += all) {
    if (!is_cut(p)) continue;
    sp.cut[kCutFirst + p] = item_start[p];
    sp.cut[kCutOrder + p] = order[p];
    if (!is_cut(p + 1)) {
      sp.cut[0] = static_cast<int32_t>(p + 1);
      sp.cut[kCutFirst + p + 1] = item_start[p + 1];
    }
  }
}

// ------------------------------------------------------------------ host side
// Most items (without cuts) of a call: every request but the last few tiles full.
inline int64_t span_most_items(const gc_kv_pool* pool, int64_t rows, int64_t batch, int num_q_heads) {
  const int64_t G = num_q_heads / pool->cfg.num_kv_heads;
  return pool->cfg.num_kv_heads * ((rows * G + (kSpanRows - 1) * batch) / kSpanRows);
}

// The workspace of a call: where its parts are, in bytes from its start.
struct SpanSpace {
  int64_t pieces, stride;
  size_t front, ml, o, end;
};
inline SpanSpace span_space(const gc_kv_pool* pool, int64_t rows, int64_t batch, int64_t max_blocks,
                            int num_q_heads, bool shared) {
  SpanSpace s{};
  const auto& c = pool->cfg;
  const int64_t G = num_q_heads / c.num_kv_heads;
  const int64_t items = span_most_items(pool, rows, batch, num_q_heads);
  const int64_t steps = (max_blocks * c.page_size + 127) / 128;
  const int64_t parts = (steps + kSpanMinSteps - 1) / kSpanMinSteps;  // of an item, at most
  const int64_t workers = c.head_dim == 128 ? pool->num_sms / 2 : pool->num_sms;
  // a plan of r rounds has at most r * workers parts more than items; where only cut
  // items count, each has two parts or more, so at most twice the equal shares
  int64_t pieces = items + kSpanRounds * workers;
  if (!shared && pieces > 2 * kSpanRounds * workers) pieces = 2 * kSpanRounds * workers;
  if (pieces > items * parts) pieces = items * parts;
  if (!shared && parts <= 1) pieces = 0;
  s.pieces = pieces;
  s.stride = rows * G < kSpanRows ? rows * G : kSpanRows;
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  s.front = 0;
  s.ml = up(shared ? static_cast<size_t>(rows) * sizeof(int4) : kCutWords * sizeof(int32_t));
  s.o = up(s.ml + static_cast<size_t>(s.pieces) * s.stride * sizeof(float2));
  s.end = up(s.o + static_cast<size_t>(s.pieces) * s.stride * c.head_dim * sizeof(float));
  if (!shared && s.pieces == 0) s.end = 0;
  return s;
}

inline SpanGeom span_geom(const SpanSpace& s, int64_t cap, bool shared, void* workspace) {
  uint8_t* w = static_cast<uint8_t*>(workspace);
  SpanGeom g{};
  g.cap = static_cast<int32_t>(cap);
  g.pieces = static_cast<int32_t>(s.pieces);
  g.stride = static_cast<int32_t>(s.stride);
  g.shared = shared ? 1 : 0;
  g.prior = shared ? reinterpret_cast<int4*>(w) : nullptr;
  g.cut = shared ? nullptr : reinterpret_cast<int32_t*>(w);
  g.ml = reinterpret_cast<float2*>(w + s.ml);
  g.o = reinterpret_cast<float*>(w + s.o);
  return g;
}

}  // namespace gc

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
//    Where requests have several row tiles over more keys than the L2 holds, the units go
//    tile by tile, all heads of a tile and then the next tile, and each such run begins
//    with a share (aligned): the workers of a request's tiles then read the same keys at
//    the same time, from memory once (questions of 43 tokens, 64/8 heads, on 131072 states:
//    440 us where the tiles of a head follow each other, 385 so).
#pragma once

#include "decode_mma.cuh"
#include "gc_internal.cuh"
#include "own_keys.h"
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
  int32_t weight;  // time of 128 own keys and a kv head on one SM, in 1/16 of a unit
  int32_t start;   // units that the own side takes beyond (its last merges)
};

constexpr int kSpanRows = 256;      // q rows of an item
constexpr int kSpanRequests = 512;  // most requests of a call that is cut into shares
// An item costs about this many steps beyond its own (its first scores, the last
// product and the results); writing the pieces and joining them takes about kSpanJoin.
constexpr int kSpanLead = 2;
constexpr int kSpanJoin = 12;
constexpr int kSpanMinShare = 4;
constexpr int kSpanInL2 = 1024;  // steps and kv heads whose K and V stay in the L2: 64 MB at d = 128

struct SpanGeom {
  int32_t cap;      // keys a block-table row can hold
  int32_t workers;  // CTAs (pairs) that take items
  int32_t stride;   // rows of a slot
  int32_t cuts;     // items may be cut
  int32_t shared;   // requests are groups (new_lens is not given); whole items' results
                    // go to `whole`, not to the output
  int32_t* plan;    // [0] units of a share, 0: whole items, [1] workers that have one
  int4* cuts_at;    // cross attention: per share, see SpanCutItem
  int4* prior;      // shared: per request, see SpanPrior
  DecodeParts whole;  // shared: [request][q head]
  float2* ml;       // [2 * workers][stride]: reference maximum, sum
  float* o;         // [2 * workers][stride][d]
};

// The cut item that begins in a worker's share, as two int4: shares c0 (this one) to c1
// (-1: there is none), slot of the first piece, kv head and tile; then first token and number of
// tokens of its request.
struct SpanCutItem {
  int32_t c1, first, g, tile, cu, n, unused[2];
};

__device__ __forceinline__ int span_steps(int T) { return T > 0 ? ((T - 1) >> 7) + 1 : 0; }
__device__ __forceinline__ int span_tiles(int n, int G) {
  return (n * G + kSpanRows - 1) / kSpanRows;
}

// How the work is dealt out: units of a share (0: whole items), and whether the runs of a
// request's tiles begin with shares.
struct SpanDeal {
  int share, aligned;
};
// Units of an item, and of one tile's items of a request.
__device__ __forceinline__ int span_per(int steps) { return steps + kSpanLead; }
__device__ __forceinline__ int span_run(SpanDeal deal, int Hkv, int steps) {
  const int run = Hkv * span_per(steps);
  return deal.aligned ? (run + deal.share - 1) / deal.share * deal.share : run;
}

// A request of a shared prefix, as an int4: its G rows of kv head g are rows
// [row, row + G) of the group's, in the item whose first unit is unit + g * span_per(steps).
// steps: of the item; 0: no shared keys, -1: the request is skipped.
struct SpanPrior {
  int32_t unit, unused, steps, row;  // (16 bytes: one load)
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
// All requests of a call, held in shared memory (three words each) where there are at
// most kSpanRequests: every role looks them up, and each look-up in global memory was a
// latency in front of the first product (prologue 3.7 us, with them held 2).
struct SpanRequests {
  const SpanGeom& sp;
  const int32_t *lens, *new_lens, *cu;
  int batch, total_new;
  int* held;

  // every thread of a CTA of `threads`; true in those that saw a bad request
  __device__ __forceinline__ bool hold(int threads) const {
    bool bad = false;
    for (int b = threadIdx.x; b < batch; b += threads) {
      const SpanRequest r = span_request(sp, b, total_new, lens, new_lens, cu);
      bad |= r.bad;
      if (batch > kSpanRequests) continue;
      held[b] = r.T;
      held[kSpanRequests + b] = r.n;
      held[2 * kSpanRequests + b] = r.cu;
    }
    return bad;
  }
  __device__ __forceinline__ SpanRequest operator()(int b) const {
    if (batch > kSpanRequests) return span_request(sp, b, total_new, lens, new_lens, cu);
    return {held[kSpanRequests + b], held[b], held[2 * kSpanRequests + b], false};
  }
};
constexpr size_t kSpanHeldBytes = 3 * kSpanRequests * sizeof(int);

// The place of a request's items in work order; start: first unit (shares) or item.
__device__ __forceinline__ int span_place(const int* start, int batch, int u) {
  int lo = 0, hi = batch;  // the last place whose start is <= u
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (start[mid] <= u) lo = mid; else hi = mid;
  }
  return lo;
}

// The least share, from `share` on, with which aligned runs need at most `workers` of them;
// 0 if it is not found soon.  By one warp.
__device__ inline int span_aligned_share(int share, int workers, int batch, int Hkv, int G,
                                         const SpanRequests& request) {
  for (int tries = 0; tries < 8; ++tries) {
    long long need = 0;
    for (int b = threadIdx.x & 31; b < batch; b += 32) {
      const SpanRequest r = request(b);
      const int st = r.n > 0 ? span_steps(r.T) : 0;
      if (st > 0)
        need += static_cast<long long>(span_tiles(r.n, G)) *
                ((Hkv * span_per(st) + share - 1) / share);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) need += __shfl_xor_sync(0xffffffffu, need, o);
    if (need <= workers) return share;
    if (need >= 2ll * workers) return 0;
    share += static_cast<int>(share * (need - workers) / (2 * workers)) + 1;
  }
  return 0;
}

// How a call is dealt out, and the workers that take part (-1: the units are too many),
// worked out by one warp; every CTA comes to the same answer.  start: each place's first item.
// kOwn: the other workers decode so many own keys, as OwnDecode says (then shares always).
struct SpanPlan {
  SpanDeal deal;
  int workers;
};
template <bool kOwn>
__device__ inline SpanPlan span_plan(const SpanGeom& sp, int batch, int Hkv, int G,
                                     long long own_keys, const OwnDecode& own, int sms_per_worker,
                                     const int* start, const int16_t* order,
                                     const SpanRequests& request) {
  if (!sp.cuts || batch > kSpanRequests) return {{0, 0}, sp.workers};
  const int lane = threadIdx.x & 31;
  long long units = 0, per_tile = 0;
  int least = INT32_MAX, most = 0, tiles = 0;
  for (int b = lane; b < batch; b += 32) {
    const SpanRequest r = request(b);
    const int st = r.n > 0 ? span_steps(r.T) : 0;
    if (st == 0) continue;
    const int t = span_tiles(r.n, G);
    per_tile += static_cast<long long>(Hkv) * span_per(st);
    units += static_cast<long long>(Hkv) * t * span_per(st);
    least = min(least, span_per(st));
    most = max(most, span_per(st));
    tiles = max(tiles, t);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    units += __shfl_xor_sync(0xffffffffu, units, o);
    per_tile += __shfl_xor_sync(0xffffffffu, per_tile, o);
  }
  tiles = __reduce_max_sync(0xffffffffu, tiles);
  // K and V more than half of the L2, and several tiles to read them
  const bool apart = tiles > 1 && per_tile > kSpanInL2;
  if constexpr (kOwn) {
    if (units == 0) return {{kSpanMinShare, 0}, 0};
    if (units >= (1ll << 30)) return {{kSpanMinShare, 0}, -1};  // (see span_scan)
    // The number w of workers for which both sides take as long,
    //     u / w = o / (W - w) + s,
    // with u units, W workers in all, o the own keys' time if they had one worker's SMs and
    // s (own.start > 0) what their side takes beyond:
    //     s w^2 - (s W + u + o) w + u W = 0;
    // the smaller root, as below W.
    const int all = static_cast<int>(units);
    const float W = static_cast<float>(sp.workers), u = static_cast<float>(all);
    const float o = static_cast<float>(own_keys) * Hkv * own.weight /
                    (128.f * 16.f * sms_per_worker);
    const float h = 0.5f * (own.start * W + u + o);
    const float w = u * W / (h + sqrtf(fmaxf(0.f, h * h - own.start * u * W)));
    // One more than that: shares are whole units, and the span side too long costs more
    // than a worker less on the other.  (One at least for own keys, and no share below the
    // least.)
    int n = min(static_cast<int>(w + 1.5f), all / kSpanMinShare);
    n = max(1, min(n, sp.workers - 1));
    const int share = max((all + n - 1) / n, kSpanMinShare);
    const int aligned = apart ? span_aligned_share(share, n, batch, Hkv, G, request) : 0;
    if (aligned > 0 && aligned <= share + share / 8) return {{aligned, 1}, n};
    return {{share, 0}, n};
  }
  if (units == 0 || units + sp.workers >= (1ll << 30)) return {{0, 0}, sp.workers};  // (32-bit units)
  // Time in steps: of whole items, longest first, against equal shares and their join.  Of
  // whole items at least r + 1 times the length of item r * workers, for every r; lane r.
  // Shares whose tiles read K and V apart must gain an eighth besides (8 x 1024 tokens of
  // 64/8 heads over 8192 states: whole items 1440 us, shares 1640).
  const int even = (static_cast<int>(units) + sp.workers - 1) / sp.workers;
  const long long nth = static_cast<long long>(lane) * sp.workers;
  int whole = 0;
  if (nth < start[batch]) {
    const int p = span_place(start, batch, static_cast<int>(nth));
    whole = (lane + 1) * span_per(span_steps(request(order[p]).T));
  }
  const long long rounds = (start[batch] + sp.workers - 1ll) / sp.workers;
  const int end = even + __reduce_min_sync(0xffffffffu, least);  // as the shortest end last
  whole = max(__reduce_max_sync(0xffffffffu, whole),
              static_cast<int>(min(static_cast<long long>(end),
                                   rounds * __reduce_max_sync(0xffffffffu, most))));
  const int share = max(even, kSpanMinShare);
  if (share + kSpanJoin >= whole) return {{0, 0}, sp.workers};
  int cost = share + (apart ? share / 8 : 0);
  const int aligned = apart ? span_aligned_share(share, sp.workers, batch, Hkv, G, request) : 0;
  const bool align = aligned > 0 && aligned < cost;
  if (align) cost = aligned;
  if (cost + kSpanJoin >= whole) return {{0, 0}, sp.workers};
  return {{align ? aligned : share, align ? 1 : 0}, sp.workers};
}

// The own keys of the requests behind shared prefixes, as the division of the SMs counts
// them (summed over a CTA's threads; cleared before).  A request of T costs T + 256 keys,
// longer ones up to 1024 more (2 T between), or T + 48 where decode_cta takes a pair per
// warp (all short, and enough of them).  This and OwnDecode's two figures were fitted to 18
// (d = 128) and 15 (d = 64) calls of 12 to 512 requests with 30 to 6000 own keys, timed with
// the workers divided in every way: 2.1 and 2.6 % on average above the best division, 8 and
// 11 % at most (with up to 768 keys for all alike, and s = -5: 10 and 8.5 %, 38 and 30 %).
struct SpanOwn {
  unsigned long long keys;
  int by_warp, longest, valid;

  __device__ __forceinline__ void clear() { *this = SpanOwn{0, 0, 0, 0}; }
  __device__ __forceinline__ void count(const OwnDecode& own, int threads) {
    const int cap = own.geo.max_blocks << own.geo.ps_shift;
    for (int b = threadIdx.x; b < own.geo.batch; b += threads) {
      const int T = ld_plain(own.lens + b);
      if (!own_keys_count(T, cap)) continue;
      keys += static_cast<unsigned long long>(own_keys_cost(T));
      by_warp += own_keys_cost_by_warp(T, dec::kShort);
      longest = max(longest, T);
      ++valid;
    }
  }
  __device__ __forceinline__ void add_to(SpanOwn* sum) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) keys += __shfl_xor_sync(0xffffffffu, keys, o);
    by_warp = __reduce_add_sync(0xffffffffu, by_warp);
    longest = __reduce_max_sync(0xffffffffu, longest);
    valid = __reduce_add_sync(0xffffffffu, valid);
    if ((threadIdx.x & 31) == 0 && valid > 0) {
      atomicAdd(&sum->keys, keys);
      atomicAdd(&sum->by_warp, by_warp);
      atomicMax(&sum->longest, longest);
      atomicAdd(&sum->valid, valid);
    }
  }
  // (decode_cta's rule, as if every CTA were on the own side)
  __device__ __forceinline__ long long cost(int Hkv) const {
    const bool warps = longest <= dec::kShort &&
                       static_cast<long long>(valid) * Hkv >= 6ll * gridDim.x;
    return warps ? by_warp : static_cast<long long>(keys);
  }
};

// Work order of up to 32 requests, longest first (ties by number), by one warp.
__device__ __forceinline__ void span_rank32(const SpanRequests& request, int16_t* order) {
  const int lane = threadIdx.x & 31, T = lane < request.batch ? request(lane).T : INT32_MIN;
  int rank = 0;
  for (int o = 0; o < request.batch; ++o) {
    const int x = __shfl_sync(0xffffffffu, T, o);
    rank += x > T || (x == T && o < lane);
  }
  if (lane < request.batch) order[rank] = static_cast<int16_t>(lane);
  __syncwarp();
}

// Worker's units [first, end) of its share.
__device__ __forceinline__ void span_share(SpanDeal deal, int worker, int units, int& first,
                                           int& end) {
  const int64_t u = static_cast<int64_t>(worker) * deal.share;
  first = static_cast<int>(min(u, static_cast<int64_t>(units)));
  end = static_cast<int>(min(u + deal.share, static_cast<int64_t>(units)));
}

// The work of a worker at unit u of its share, or (share 0) item u.  nt 0: there is none
// left in the share.  slot: of its pieces, -1 if it is a whole item; next: the unit after.
struct SpanPiece {
  int b, g, tile, n, T, cu, j0, nt, slot, next;
};
__device__ __forceinline__ SpanPiece span_piece(int u, SpanDeal deal, int worker, int batch,
                                                const int* start, const int16_t* order, int Hkv,
                                                int G, const SpanRequests& request) {
  SpanPiece w;
  const int p = span_place(start, batch, u);
  w.b = batch <= kSpanRequests ? order[p] : p;
  const SpanRequest r = request(w.b);
  w.n = r.n;
  w.T = r.T;
  w.cu = r.cu;
  const int steps = span_steps(r.T), tiles = span_tiles(r.n, G), local = u - start[p];
  if (deal.share == 0) {
    // the tiles that read the same keys one after the other
    w.g = local / tiles;
    w.tile = local - w.g * tiles;
    w.j0 = 0;
    w.nt = steps;
    w.slot = -1;
    w.next = u + 1;
    return w;
  }
  int first, end;
  span_share(deal, worker, start[batch], first, end);
  const int per = span_per(steps), run = span_run(deal, Hkv, steps);
  w.tile = local / run;
  const int in_run = local - w.tile * run;
  w.g = in_run / per;
  const int off = in_run - w.g * per, to = min(per, off + (end - u));
  w.j0 = max(0, off - kSpanLead);
  w.nt = max(0, to - kSpanLead - w.j0);
  w.slot = w.nt < steps ? 2 * worker + (u == first ? 0 : 1) : -1;
  w.next = u + to - off;
  if (w.g >= Hkv) {  // what fills a run's last share
    w.nt = 0;
    w.next = end;
  }
  return w;
}

// Exclusive scan, by one warp, of the places' items (share 0) or units into start,
// and each request's into first_of where it is given.  False, and nothing to do, if there
// are too many for 32-bit ints: the host has checked that for requests that divide the
// rows, so some have rows in common.
__device__ inline bool span_scan(SpanDeal deal, int Hkv, int G, const int16_t* order, int* start,
                                 int* first_of, const SpanRequests& request) {
  const int lane = threadIdx.x & 31, batch = request.batch;
  long long running = 0;
  for (int p0 = 0; p0 < batch; p0 += 32) {
    const int p = p0 + lane;
    const int b = p < batch && batch <= kSpanRequests ? order[p] : p;
    long long cnt = 0;
    if (p < batch) {
      const SpanRequest r = request(b);
      const int steps = r.n > 0 ? span_steps(r.T) : 0;
      if (steps > 0)
        cnt = static_cast<long long>(span_tiles(r.n, G)) *
              (deal.share ? span_run(deal, Hkv, steps) : Hkv);
    }
    long long incl = cnt;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long y = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += y;
    }
    if (p < batch) start[p] = static_cast<int>(running + incl - cnt);
    if (p < batch && first_of) first_of[b] = static_cast<int>(running + incl - cnt);
    running += __shfl_sync(0xffffffffu, incl, 31);
  }
  const bool fits = running < INT32_MAX - 4096;  // (workers look one past it)
  if (!fits)
    for (int p = lane; p < batch; p += 32) start[p] = 0;
  if (lane == 0) start[batch] = fits ? static_cast<int>(running) : 0;
  __syncwarp();
  return fits;
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
__device__ inline void span_write_plan(const SpanGeom& sp, SpanDeal deal, int workers, int Hkv,
                                       int G, const int* start, const int16_t* order,
                                       const SpanRequests& request, int64_t me, int64_t all) {
  if (!sp.plan) return;
  if (me == 0) {
    sp.plan[0] = deal.share;
    sp.plan[1] = workers;
  }
  if (deal.share == 0 || sp.shared) return;
  const int batch = request.batch;
  for (int64_t worker = me; worker < workers; worker += all) {
    SpanCutItem x{-1, 0, 0, 0, 0, 0, {0, 0}};
    const int64_t end = (worker + 1) * deal.share;
    if (end < start[batch]) {
      // the item that the share's end lies in
      const int p = span_place(start, batch, static_cast<int>(end));
      const SpanRequest r = request(order[p]);
      const int steps = span_steps(r.T), per = span_per(steps), run = span_run(deal, Hkv, steps);
      const int local = static_cast<int>(end) - start[p], tile = local / run;
      const int in_run = local - tile * run, g = in_run / per;
      const SpanCut cut = span_cut(static_cast<int>(end) - (in_run - g * per), steps, deal.share);
      if (g < Hkv && cut.c0 == worker && cut.c1 > cut.c0)
        x = SpanCutItem{cut.c1, cut.first, g, tile, r.cu, r.n, {0, 0}};
    }
    sp.cuts_at[2 * worker] = make_int4(x.c1, x.first, x.g, x.tile);
    sp.cuts_at[2 * worker + 1] = make_int4(x.cu, x.n, 0, 0);
  }
}

// Thread `me` of `all`: the requests' rows of the groups' items.  first_of: each
// group's first unit or item.
__device__ inline void span_priors(const SpanGeom& sp, SpanDeal deal, bool fits, int Hkv, int G,
                                   const int* first_of, const SpanRequests& request, int64_t me,
                                   int64_t all) {
  for (int64_t b = me; b < request.total_new; b += all) {
    int lo = 0, hi = request.batch;  // the last group whose first request is <= b
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (ld_plain(request.cu + mid) <= b) lo = mid; else hi = mid;
    }
    const SpanRequest r = request(lo);
    SpanPrior p{0, 0, -1, 0};
    if (fits && !r.bad && b >= r.cu && b < r.cu + r.n) {
      p.steps = span_steps(r.T);
      p.row = (static_cast<int>(b) - r.cu) * G;
      if (deal.share) p.unit = first_of[lo] + p.row / kSpanRows * span_run(deal, Hkv, p.steps);
    }
    sp.prior[b] = make_int4(p.unit, 0, p.steps, p.row);
  }
}

// Thread `me` of `all` (whole warps): zeros for the rows of requests without keys.
__device__ inline void span_zeros(int Hq, int D, const SpanRequests& request, __nv_bfloat16* out,
                                  int64_t me, int64_t all) {
  const int lane = threadIdx.x & 31;
  for (int b0 = 0; b0 < request.batch; b0 += 32) {
    const bool none = b0 + lane < request.batch && request(b0 + lane).T == 0;
    uint32_t which = __ballot_sync(0xffffffffu, none);
    for (; which; which &= which - 1) {
      const SpanRequest r = request(b0 + __ffs(which) - 1);
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
  size_t plan, cuts_at, prior, whole_ml, whole_o, ml, o, end;
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
  s.plan = take(shared || s.slots ? 2 * sizeof(int32_t) : 0);
  s.cuts_at = take(shared ? 0 : s.slots * sizeof(int4));
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
  g.cuts_at = shared ? nullptr : reinterpret_cast<int4*>(w + s.cuts_at);
  g.prior = shared ? reinterpret_cast<int4*>(w + s.prior) : nullptr;
  if (shared)
    g.whole = DecodeParts{reinterpret_cast<float*>(w + s.whole_o),
                          reinterpret_cast<float2*>(w + s.whole_ml)};
  g.ml = reinterpret_cast<float2*>(w + s.ml);
  g.o = reinterpret_cast<float*>(w + s.o);
  return g;
}

}  // namespace gc

// Where a new token goes and how its heads are rotated: what the appends to 16-bit and to
// 4-bit pages share (append_rope.cu, append_q4.cu).
#pragma once

#include "gc_internal.cuh"
#include "sm103_ptx.cuh"

namespace gc {
namespace {

using ptx::pack_bf16x2;

constexpr int kBlock = 256;

struct RopeGeom {
  int32_t Hq, Hkv, ps_shift, num_pages, batch, max_blocks, layer, total_new;
  int32_t head_shift;    // units of a head, log2 (d / 16)
  int32_t rot_units;     // units of a head that are rotated (rot / 16)
  int32_t heads;         // Hq + 2 Hkv (16-bit pages)
  int32_t threads;       // of a token: ceil(heads / W) << head_shift
  int32_t interleaved, n_positions;
  int64_t q_stride, k_stride, v_stride;  // 16-byte words between tokens
};

// Where a token goes.
struct Place {
  int32_t pos;   // row of the angle table, -1: the token is skipped
  int32_t page;  // page of its K and V, -1: none
  int32_t slot;  // slot in the page
};

// By kLanes lanes for each token, 8 (whole warps together) or 1.  Each step of the search for
// its request is a load that the next one waits for, so where that is most of the call's
// time eight lanes take eight requests at once (200 tokens of as many requests, 32/8 heads:
// 4.05 -> 3.6 us; with many tokens a block's other loads hide it and the lanes' registers
// cost more, 8 x 1024 tokens 55.4 -> 57.4).
template <int kLanes>
__device__ Place look_up(int64_t t, const RopeGeom& g, const int32_t* block_table,
                         const int32_t* prefix_lens, const int32_t* cu_new_lens,
                         const int32_t* positions, int32_t* status) {
  const int lane = threadIdx.x & 31, k = lane % kLanes;
  const int64_t given = kLanes > 1 && positions ? ld_plain(positions + t) : 0;
  // request b with cu[b] <= t < cu[b+1]: last b whose start is <= t
  int lo = 0;
  if constexpr (kLanes == 1) {
    int hi = g.batch;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (ld_plain(cu_new_lens + mid) <= t) lo = mid; else hi = mid;
    }
  } else {
    for (int n = g.batch; n > 1;) {
      n = (n + kLanes - 1) / kLanes;
      const int b = lo + k * n;
      const bool before = k == 0 || (b < g.batch && ld_plain(cu_new_lens + b) <= t);
      const uint32_t all = __ballot_sync(0xffffffffu, before) >> (lane - k) & 0xffu;
      lo = min(lo + (31 - __clz(all)) * n, g.batch - 1);
    }
  }
  const int start = ld_plain(cu_new_lens + lo), end = ld_plain(cu_new_lens + lo + 1);
  const int prefix = ld_plain(prefix_lens + lo);
  Place w{-1, -1, 0};
  const bool sane = t >= start && t < end && end <= g.total_new && prefix >= 0;
  const int64_t at = prefix + (t - start);
  const int64_t pos = !positions || !sane ? at : kLanes > 1 ? given : ld_plain(positions + t);
  if (!sane || pos < 0 || pos >= g.n_positions) {
    if (k == 0) record_error(status, GC_ERR_OUT_OF_RANGE);
    return w;
  }
  w.pos = static_cast<int32_t>(pos);
  w.slot = static_cast<int32_t>(at & ((1 << g.ps_shift) - 1));
  const int64_t blk = at >> g.ps_shift;
  if (blk < g.max_blocks)
    w.page = ld_plain(block_table + static_cast<int64_t>(lo) * g.max_blocks + blk);
  if (w.page < 0 || w.page >= g.num_pages) {
    if (k == 0) record_error(status, GC_ERR_OUT_OF_RANGE);
    w.page = -1;
  }
  return w;
}

__device__ __forceinline__ float lo_f32(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float hi_f32(uint32_t v) { return __uint_as_float(v & 0xffff0000u); }

// Pair members in the same half of the two words' elements.
__device__ __forceinline__ void turn(uint32_t& x, uint32_t& y, float c0, float s0, float c1,
                                     float s1) {
  const float x0 = lo_f32(x), x1 = hi_f32(x), y0 = lo_f32(y), y1 = hi_f32(y);
  x = pack_bf16x2(fmaf(x0, c0, -(y0 * s0)), fmaf(x1, c1, -(y1 * s1)));
  y = pack_bf16x2(fmaf(y0, c0, x0 * s0), fmaf(y1, c1, x1 * s1));
}
// Neighbours: one pair to a 32-bit word.
__device__ __forceinline__ void turn(uint32_t& xy, float c, float s) {
  const float x = lo_f32(xy), y = hi_f32(xy);
  xy = pack_bf16x2(fmaf(x, c, -(y * s)), fmaf(y, c, x * s));
}

int ilog2(int x) {
  int s = 0;
  while ((1 << s) < x) ++s;
  return s;
}

}  // namespace
}  // namespace gc

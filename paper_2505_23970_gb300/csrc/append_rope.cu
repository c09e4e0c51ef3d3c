// Append of the new tokens' K and V to the paged pool with the position rotation
// on the way, and the rotated queries written for the attention that follows
// (Sec. 2.2: the new tokens' KV is stitched after the cached one).
//
// For new token t of request b, at position p and slot s = prefix_b + t, a head's
// columns are rotated in pairs (x, y), pair i by the angle whose cosine and sine
// the table holds at [p][0][i] and [p][1][i]:
//     x' = x cos - y sin,   y' = y cos + x sin
// with pairs (i, i + rot/2), or (2i, 2i + 1) when interleaved; columns from rot
// on, and V, are copied.  Products and sums are binary32, each result is rounded
// once to bf16 (the type of the pool and of the attention's q).
//
// Bound: HBM (q, k and v read once, written once) where the tokens are many, the
// chain of look-ups where they are few.
//  * A thread's unit is 16 elements of a head, two 16-byte words half a rotated
//    (or copied) section apart: with either kind of pair both members of its 8
//    pairs are in those words, and a warp's loads and stores are contiguous.
//  * The data does not depend on the look-ups, so its loads are issued first; a
//    block's tokens are then looked up (request, position, page) by one thread
//    or eight lanes each instead of by every thread.
//
// Measured: 8 x 1024 tokens of 64/8 heads of 128 (340 MB) 55.7 us, 6.1 TB/s, 0.90 of the
// copy rate (ncu: the wait for the look-ups is the longest stall); 8 tokens 6.6 us, the
// length of the call's own path on the host; 4400 ragged tokens of 32/8 heads of 64 12.4 us.
#include "append_place.cuh"

namespace gc {
namespace {

constexpr int kMinThreads = 4;  // of a token, at least: the units of a head of 64

// A thread has the units of W neighbouring heads at one place of them.
template <int W>
__global__ void __launch_bounds__(kBlock)
    append_rope_kernel(const uint4* q, uint4* q_out, const uint4* k_new, const uint4* v_new,
                       uint8_t* pool, const int32_t* block_table, const int32_t* prefix_lens,
                       const int32_t* cu_new_lens, const float* cos_sin,
                       const int32_t* positions, RopeGeom g, int32_t* status) {
  __shared__ Place places[kBlock / kMinThreads + 2];
  dependent_begin();
  const int64_t total = static_cast<int64_t>(g.total_new) * g.threads;
  const int hs = g.head_shift;
  for (int64_t base = static_cast<int64_t>(blockIdx.x) * kBlock; base < total;
       base += static_cast<int64_t>(gridDim.x) * kBlock) {
    const int64_t t0 = base / g.threads;
    const int first = static_cast<int>(base - t0 * g.threads);  // thread of token t0
    const int local = first + static_cast<int>(threadIdx.x);
    const int tl = local / g.threads, u = local - tl * g.threads;
    const int64_t t = t0 + tl;
    const int h0 = (u >> hs) * W, s = u & ((1 << hs) - 1);  // first head (q, then k, then v)
    // the unit's words: of the rotated section (n apart), of the columns after it, or of V
    const bool rotated = s < g.rot_units;
    const int n = rotated ? g.rot_units : (1 << hs) - g.rot_units;
    const int in_head = rotated ? s : g.rot_units + s;
    uint4 a[W], b[W];
#pragma unroll
    for (int w = 0; w < W; ++w) {
      int h = h0 + w;
      if (t >= g.total_new || h >= g.heads) continue;
      const uint4* src;
      if (h < g.Hq)
        src = q + t * g.q_stride;
      else if ((h -= g.Hq) < g.Hkv)
        src = k_new + t * g.k_stride;
      else
        src = v_new + t * g.v_stride, h -= g.Hkv;
      src += (h << (hs + 1)) + in_head;
      a[w] = ld_plain(src);
      b[w] = ld_plain(src + n);
    }
    const int tokens = (first + kBlock - 1) / g.threads + 1;  // of this block's threads
    __syncthreads();  // the places of the round before have been read
    const int most = static_cast<int>(min(static_cast<int64_t>(tokens), g.total_new - t0));
    constexpr int kLanes = W == 1 ? 8 : 1;
    for (int i0 = 0; i0 < most; i0 += kBlock / kLanes) {
      const int mine = i0 + static_cast<int>(threadIdx.x) / kLanes;
      if (kLanes == 1 && mine >= most) continue;
      const int i = min(mine, most - 1);
      const Place w =
          look_up<kLanes>(t0 + i, g, block_table, prefix_lens, cu_new_lens, positions, status);
      if (threadIdx.x % kLanes == 0) places[i] = w;
    }
    __syncthreads();
    if (t >= g.total_new) continue;
    const Place p = places[tl];
    if (p.pos < 0) continue;
    if (rotated && h0 < g.Hq + g.Hkv) {
      // angles of the unit's pairs: 8 in a row, or 4 of each word's
      const float4* cs = reinterpret_cast<const float4*>(
          cos_sin + static_cast<int64_t>(p.pos) * 16 * g.rot_units);
      const int i0 = g.interleaved ? s : 2 * s;
      const int i1 = g.interleaved ? s + g.rot_units : 2 * s + 1;
      const float4 c0 = ld_plain(cs + i0), c1 = ld_plain(cs + i1);
      const float4 s0 = ld_plain(cs + 2 * g.rot_units + i0), s1 = ld_plain(cs + 2 * g.rot_units + i1);
#pragma unroll
      for (int w = 0; w < W; ++w) {
        if (h0 + w >= g.Hq + g.Hkv) continue;
        if (g.interleaved) {
          turn(a[w].x, c0.x, s0.x);
          turn(a[w].y, c0.y, s0.y);
          turn(a[w].z, c0.z, s0.z);
          turn(a[w].w, c0.w, s0.w);
          turn(b[w].x, c1.x, s1.x);
          turn(b[w].y, c1.y, s1.y);
          turn(b[w].z, c1.z, s1.z);
          turn(b[w].w, c1.w, s1.w);
        } else {
          turn(a[w].x, b[w].x, c0.x, s0.x, c0.y, s0.y);
          turn(a[w].y, b[w].y, c0.z, s0.z, c0.w, s0.w);
          turn(a[w].z, b[w].z, c1.x, s1.x, c1.y, s1.y);
          turn(a[w].w, b[w].w, c1.z, s1.z, c1.w, s1.w);
        }
      }
    }
#pragma unroll
    for (int w = 0; w < W; ++w) {
      int h = h0 + w;
      if (h >= g.heads || (h >= g.Hq && p.page < 0)) continue;
      uint4* dst;
      if (h < g.Hq) {
        dst = q_out + (((t * g.Hq + h) << (hs + 1)) + in_head);
      } else {
        const int kv = h < g.Hq + g.Hkv ? 0 : 1;
        h -= g.Hq + kv * g.Hkv;
        const int64_t row =
            ((((static_cast<int64_t>(g.layer) * 2 + kv) * g.num_pages + p.page) * g.Hkv + h)
             << g.ps_shift) + p.slot;
        dst = reinterpret_cast<uint4*>(pool) + ((row << (hs + 1)) + in_head);
      }
      dst[0] = a[w];
      dst[n] = b[w];
    }
  }
}

}  // namespace

gc_status launch_append_rope(const gc_kv_pool* pool, const RopeArgs& a, cudaStream_t stream) {
  const auto& cfg = pool->cfg;
  RopeGeom g;
  g.Hq = a.num_q_heads;
  g.Hkv = cfg.num_kv_heads;
  g.ps_shift = ilog2(cfg.page_size);
  g.num_pages = cfg.num_pages;
  g.batch = a.batch;
  g.max_blocks = a.max_blocks;
  g.layer = a.layer;
  g.total_new = a.total_new_tokens;
  g.head_shift = ilog2(cfg.head_dim / 16);
  g.rot_units = a.rot_dim / 16;
  g.heads = g.Hq + 2 * g.Hkv;
  g.interleaved = a.interleaved ? 1 : 0;
  g.n_positions = a.n_positions;
  g.q_stride = a.q_stride / 8;
  g.k_stride = a.k_stride / 8;
  g.v_stride = a.v_stride / 8;
  // Two units a thread, which then reads the angles once for both, where one each would
  // not be resident at once (8 x 1024 tokens of 64/8 heads of 128: one 76.5 us, two 55.8,
  // 6.1 TB/s, four 55.5, eight 64; 4400 tokens of 32/8 heads of 64: 15.4, 12.7, 14.1,
  // 15.8); a call of few tokens is latency alone.
  const bool few = (static_cast<int64_t>(g.total_new) * g.heads << g.head_shift) <=
                   static_cast<int64_t>(pool->num_sms) * 2048;
  const int W = few ? 1 : 2;
  g.threads = (g.heads + W - 1) / W << g.head_shift;
  const int64_t blocks = (static_cast<int64_t>(g.total_new) * g.threads + kBlock - 1) / kBlock;
  const int64_t cap = static_cast<int64_t>(pool->num_sms) * 32;
  const unsigned grid = static_cast<unsigned>(blocks < cap ? blocks : cap);
  const cudaError_t e = launch_dependent(
      few ? append_rope_kernel<1> : append_rope_kernel<2>, grid, kBlock, 0, stream,
      static_cast<const uint4*>(a.q), static_cast<uint4*>(a.q_out),
      static_cast<const uint4*>(a.k_new), static_cast<const uint4*>(a.v_new), pool->data,
      a.block_table, a.prefix_lens, a.cu_new_lens, a.cos_sin, a.positions, g, pool->status);
  if (e != cudaSuccess) return cuda_fail(e, "gc_kv_append_rope: kernel launch");
  return GC_OK;
}

}  // namespace gc

// Append of the new tokens to 4-bit pages as their projection gives them: q and k are
// rotated to their positions, q is written for the attention that follows, k and v are
// quantised as they are written (Sec. 2.2: the new tokens' KV is stitched after the cached
// one; Sec. 6.1: the 70B runs keep what they can in few bits).
//
// The rotation and its rounding to bf16 are append_rope.cu's, the format q4_format.cuh's; a
// key is rounded to bf16 between the two, so that the page holds what packing the 16-bit
// page would give, bit for bit.
//
// Bound: HBM where the tokens are many (q, k and v read once, q and 0.28 of k and v
// written), the chain of look-ups where they are few.  The first blocks have the rows of
// k and v: four lanes a row, each with 8 columns of every group, so that a group's maximum
// is two shuffles, both members of a pair of neighbours are in one lane and a lane's codes
// are one store.  A pair in halves is met by reading the other half's 8 columns too (from
// the L1: the row's other lanes read them).  The other blocks turn q as append_rope.cu does.
//
// Measured: 8 x 1024 tokens of 64/8 heads of 128 (311 MB) 57 us, 5.5 TB/s, 0.81 of the copy
// rate (ncu: the wait for the look-ups and for the loads before them, as in append_rope.cu,
// which moves 340 MB in 56); 8 tokens 6.4 us; 4400 ragged tokens of 32/8 heads of 64 11 us.
#include "append_place.cuh"
#include "q4_format.cuh"

namespace gc {
namespace {

constexpr int kRows = kBlock / 4;  // of k and v in a block

__device__ __forceinline__ void neighbours8(uint4& x, const float4& c, const float4& s) {
  turn(x.x, c.x, s.x);
  turn(x.y, c.y, s.y);
  turn(x.z, c.z, s.z);
  turn(x.w, c.w, s.w);
}

// x c + sign y s, in pairs of columns
__device__ __forceinline__ uint32_t half_pair(uint32_t x, uint32_t y, float sign, float c0,
                                              float s0, float c1, float s1) {
  return pack_bf16x2(fmaf(lo_f32(x), c0, sign * (lo_f32(y) * s0)),
                     fmaf(hi_f32(x), c1, sign * (hi_f32(y) * s1)));
}
__device__ __forceinline__ void halves8(uint4& x, const uint4& y, float sign, const float4* c,
                                        const float4* s) {
  const float4 c0 = ld_plain(c), c1 = ld_plain(c + 1), s0 = ld_plain(s), s1 = ld_plain(s + 1);
  x.x = half_pair(x.x, y.x, sign, c0.x, s0.x, c0.y, s0.y);
  x.y = half_pair(x.y, y.y, sign, c0.z, s0.z, c0.w, s0.w);
  x.z = half_pair(x.z, y.z, sign, c1.x, s1.x, c1.y, s1.y);
  x.w = half_pair(x.w, y.w, sign, c1.z, s1.z, c1.w, s1.w);
}

// The places of tokens t0 ... t0 + count - 1, by the whole block.
template <int kLanes>
__device__ void look_up_all(Place* places, int64_t t0, int count, const RopeGeom& g,
                            const int32_t* table, const int32_t* prefix_lens,
                            const int32_t* cu_new_lens, const int32_t* positions,
                            int32_t* status) {
  __syncthreads();  // the places of the round before have been read
  const int most = static_cast<int>(min(static_cast<int64_t>(count), g.total_new - t0));
  for (int i0 = 0; i0 < most; i0 += kBlock / kLanes) {
    const int mine = i0 + static_cast<int>(threadIdx.x) / kLanes;
    if (kLanes == 1 && mine >= most) continue;
    const int i = min(mine, most - 1);
    const Place w = look_up<kLanes>(t0 + i, g, table, prefix_lens, cu_new_lens, positions, status);
    if (threadIdx.x % kLanes == 0) places[i] = w;
  }
  __syncthreads();
}

// The rows of k and v: row = token * 2 Hkv + head, keys first.
template <int GR, int kLanes>
__device__ __forceinline__ void kv_rows(Place* places, int block, int blocks, const uint4* k_new,
                                        const uint4* v_new, const Q4Geom& q4,
                                        const int32_t* table, const int32_t* prefix_lens,
                                        const int32_t* cu_new_lens, const float* cos_sin,
                                        const int32_t* positions, const RopeGeom& g,
                                        int32_t* status) {
  const int heads = 2 * g.Hkv, q = threadIdx.x & 3;
  const int rot = 16 * g.rot_units, half = rot / 2;
  const int64_t rows = static_cast<int64_t>(g.total_new) * heads;
  for (int64_t base = static_cast<int64_t>(block) * kRows; base < rows;
       base += static_cast<int64_t>(blocks) * kRows) {
    const int64_t t0 = base / heads;
    const int local = static_cast<int>(base - t0 * heads) + static_cast<int>(threadIdx.x >> 2);
    const int tl = local / heads;
    int h = local - tl * heads;
    const int64_t t = t0 + tl;
    const bool is_k = h < g.Hkv;
    if (!is_k) h -= g.Hkv;
    uint4 x[GR];
#pragma unroll
    for (int i = 0; i < GR; ++i) x[i] = make_uint4(0, 0, 0, 0);
    const uint4* src =
        (is_k ? k_new + t * g.k_stride : v_new + t * g.v_stride) + h * (4 * GR) + q;
    if (t < g.total_new) {
#pragma unroll
      for (int i = 0; i < GR; ++i) x[i] = ld_plain(src + 4 * i);
    }
    const int last = static_cast<int>(base - t0 * heads) + kRows - 1;
    look_up_all<kLanes>(places, t0, last / heads + 1, g, table, prefix_lens, cu_new_lens,
                        positions, status);
    const Place p = t < g.total_new ? places[tl] : Place{-1, -1, 0};
    const bool write = p.pos >= 0 && p.page >= 0;
    if (is_k && write) {
      const float* cs = cos_sin + static_cast<int64_t>(p.pos) * rot;
#pragma unroll
      for (int i = 0; i < GR; ++i) {
        const int c0 = 32 * i + 8 * q;
        if (c0 >= rot) continue;
        if (g.interleaved) {
          const float4* c = reinterpret_cast<const float4*>(cs + c0 / 2);
          neighbours8(x[i], ld_plain(c), ld_plain(c + half / 4));
        } else {
          const bool second = c0 >= half;
          const float4* c = reinterpret_cast<const float4*>(cs + c0 - (second ? half : 0));
          const uint4 y = ld_plain(src + 4 * i + (second ? -half : half) / 8);
          halves8(x[i], y, second ? 1.f : -1.f, c, c + half / 4);
        }
      }
    }
    uint8_t* head = write ? q4_head(q4, g.layer, is_k ? 0 : 1, p.page, h) : q4.cache;
    q4::store_row<GR>(x, is_k, head + p.slot * (16 * GR),
                      head + (q4.ps * (16 * GR) + p.slot * (2 * GR)), write);
  }
}

// A thread has the units of W neighbouring q heads at one place of them.
template <int W>
__device__ __forceinline__ void q_units(Place* places, int block, int blocks, const uint4* q,
                                        uint4* q_out, const int32_t* table,
                                        const int32_t* prefix_lens, const int32_t* cu_new_lens,
                                        const float* cos_sin, const int32_t* positions,
                                        const RopeGeom& g, int32_t* status) {
  constexpr int kLanes = W == 1 ? 8 : 1;
  const int64_t total = static_cast<int64_t>(g.total_new) * g.threads;
  const int hs = g.head_shift;
  for (int64_t base = static_cast<int64_t>(block) * kBlock; base < total;
       base += static_cast<int64_t>(blocks) * kBlock) {
    const int64_t t0 = base / g.threads;
    const int first = static_cast<int>(base - t0 * g.threads);
    const int local = first + static_cast<int>(threadIdx.x);
    const int tl = local / g.threads, u = local - tl * g.threads;
    const int64_t t = t0 + tl;
    const int h0 = (u >> hs) * W, s = u & ((1 << hs) - 1);
    // the unit's words: of the rotated section (n apart) or of the columns after it
    const bool rotated = s < g.rot_units;
    const int n = rotated ? g.rot_units : (1 << hs) - g.rot_units;
    const int in_head = rotated ? s : g.rot_units + s;
    uint4 a[W], b[W];
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const int h = h0 + w;
      if (t >= g.total_new || h >= g.Hq) continue;
      const uint4* src = q + t * g.q_stride + ((h << (hs + 1)) + in_head);
      a[w] = ld_plain(src);
      b[w] = ld_plain(src + n);
    }
    look_up_all<kLanes>(places, t0, (first + kBlock - 1) / g.threads + 1, g, table, prefix_lens,
                        cu_new_lens, positions, status);
    if (t >= g.total_new) continue;
    const Place p = places[tl];
    if (p.pos < 0) continue;
    if (rotated) {
      const float4* cs = reinterpret_cast<const float4*>(
          cos_sin + static_cast<int64_t>(p.pos) * 16 * g.rot_units);
      const int i0 = g.interleaved ? s : 2 * s;
      const int i1 = g.interleaved ? s + g.rot_units : 2 * s + 1;
      const float4 c0 = ld_plain(cs + i0), c1 = ld_plain(cs + i1);
      const float4 s0 = ld_plain(cs + 2 * g.rot_units + i0);
      const float4 s1 = ld_plain(cs + 2 * g.rot_units + i1);
#pragma unroll
      for (int w = 0; w < W; ++w) {
        if (h0 + w >= g.Hq) continue;
        if (g.interleaved) {
          neighbours8(a[w], c0, s0);
          neighbours8(b[w], c1, s1);
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
      const int h = h0 + w;
      if (h >= g.Hq) continue;
      uint4* dst = q_out + (((t * g.Hq + h) << (hs + 1)) + in_head);
      dst[0] = a[w];
      dst[n] = b[w];
    }
  }
}

// (Five blocks an SM: the registers that the rows of k and v would take otherwise leave
// room for three, and too few loads of q are under way then: 8 x 1024 tokens of 64/8 heads
// of 128 take 73 us, four blocks 62, five 57, six, with spills, 58.)
template <int GR, int W>
__global__ void __launch_bounds__(kBlock, 5)
    append_q4_kernel(const uint4* q, uint4* q_out, const uint4* k_new, const uint4* v_new,
                     Q4Geom q4, const int32_t* table, const int32_t* prefix_lens,
                     const int32_t* cu_new_lens, const float* cos_sin, const int32_t* positions,
                     RopeGeom g, int kv_blocks, int32_t* status) {
  // tokens of a block: 256 threads with at least 4 units of a token's q heads, or 64 rows
  // with at least 2 of its heads
  __shared__ Place places[kBlock / 4 + 2];
  dependent_begin();
  const int block = static_cast<int>(blockIdx.x);
  if (block < kv_blocks)
    kv_rows<GR, W == 1 ? 8 : 1>(places, block, kv_blocks, k_new, v_new, q4, table, prefix_lens,
                                cu_new_lens, cos_sin, positions, g, status);
  else
    q_units<W>(places, block - kv_blocks, static_cast<int>(gridDim.x) - kv_blocks, q, q_out,
               table, prefix_lens, cu_new_lens, cos_sin, positions, g, status);
}

}  // namespace

size_t q4_bytes(const gc_pool_config& c, int32_t pages) {
  return static_cast<size_t>(c.num_layers) * 2 * pages * c.num_kv_heads *
         q4_head_bytes(c.head_dim, c.page_size);
}

Q4Geom q4_geom(const gc_kv_pool* pool, const Q4Cache& cache) {
  const auto& cfg = pool->cfg;
  return Q4Geom{const_cast<uint8_t*>(cache.data), q4_head_bytes(cfg.head_dim, cfg.page_size),
                cache.pages, cfg.num_kv_heads, cfg.page_size, ilog2(cfg.page_size)};
}

gc_status launch_append_q4(const gc_kv_pool* pool, const RopeArgs& a, const Q4Cache& cache,
                           cudaStream_t stream) {
  const auto& cfg = pool->cfg;
  RopeGeom g{};
  g.Hq = a.num_q_heads;
  g.Hkv = cfg.num_kv_heads;
  g.ps_shift = ilog2(cfg.page_size);
  g.num_pages = cache.pages;
  g.batch = a.batch;
  g.max_blocks = a.max_blocks;
  g.layer = a.layer;
  g.total_new = a.total_new_tokens;
  g.head_shift = ilog2(cfg.head_dim / 16);
  g.rot_units = a.rot_dim / 16;
  g.interleaved = a.interleaved ? 1 : 0;
  g.n_positions = a.n_positions;
  g.q_stride = a.q_stride / 8;
  g.k_stride = a.k_stride / 8;
  g.v_stride = a.v_stride / 8;
  // (the rule and its reason: append_rope.cu)
  const int64_t heads = g.Hq + 2 * static_cast<int64_t>(g.Hkv);
  const bool few = (g.total_new * heads << g.head_shift) <=
                   static_cast<int64_t>(pool->num_sms) * 2048;
  const int W = few ? 1 : 2;
  g.threads = (g.Hq + W - 1) / W << g.head_shift;
  const int64_t cap = static_cast<int64_t>(pool->num_sms) * 32;
  const int64_t kv = (static_cast<int64_t>(g.total_new) * 2 * g.Hkv + kRows - 1) / kRows;
  const int64_t qs = (static_cast<int64_t>(g.total_new) * g.threads + kBlock - 1) / kBlock;
  const int kv_blocks = static_cast<int>(kv < cap ? kv : cap);
  const unsigned grid = static_cast<unsigned>(kv_blocks + (qs < cap ? qs : cap));
  auto kernel = cfg.head_dim == 128 ? few ? append_q4_kernel<4, 1> : append_q4_kernel<4, 2>
                : few               ? append_q4_kernel<2, 1>
                                    : append_q4_kernel<2, 2>;
  const cudaError_t e = launch_dependent(
      kernel, grid, kBlock, 0, stream, static_cast<const uint4*>(a.q),
      static_cast<uint4*>(a.q_out), static_cast<const uint4*>(a.k_new),
      static_cast<const uint4*>(a.v_new), q4_geom(pool, cache), a.block_table, a.prefix_lens,
      a.cu_new_lens, a.cos_sin, a.positions, g, kv_blocks, pool->status);
  if (e != cudaSuccess) return cuda_fail(e, "gc_kv_append_rope_q4: kernel launch");
  return GC_OK;
}

}  // namespace gc

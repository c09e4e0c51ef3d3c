// A warp's work on keys in 4-bit pages (decode_q4.cu says how the kernel works).
//
// The products are decode_mma.cu's, S^T = K Q^T and O^T += V^T P^T by m16n8k16, with the
// codes as operands just as they are stored: masking a word leaves, in each 16-bit half, a
// nibble at bits 0-3 or 4-7 and zeros.  As bf16 that is the subnormal number
//     u 2^-133 or u 2^-129,  u = c + 8
// (the patterns up to 0xff are evenly spaced), which the tensor cores multiply exactly.  A
// word of 8 codes so costs one shift and four masks, no conversion and no offset:
//  * the weight 16 of the second kind is taken out of the other operand (K: Q's columns
//    are divided by 16) or of the result's row (V: row r + 8 of a tile), exactly;
//  * the offset 8 starts the accumulators of S (-8 sum q over the group, worked out once
//    per piece) and is one more product with a constant operand for O;
//  * S is scaled group by group in binary32, S += s_g D_g; P is scaled by V's s_g before
//    its product, P s_g rounded to bf16 (2^-9 of a term, as P itself is).
// Powers of two keep everything in range: Q's columns are brought to 2^60 at the most, P
// is 2^90 2^(x - m), and both leave again exactly.
#pragma once

#include "decode_mma.cuh"
#include "q4_format.cuh"

namespace gc {
namespace {
namespace dec {

constexpr int kQTop = 60;          // exponent of a column's largest |q|
constexpr float kPBias = 90.0f;    // P is 2^kPBias at the reference maximum
constexpr float kRaise4 = 8.0f;    // scores this far above it raise it
constexpr uint32_t kLowNibbles = 0x000f000fu, kHighNibbles = 0x00f000f0u;

__device__ __forceinline__ float pow2(int e) {  // -126 <= e <= 127
  return __uint_as_float(static_cast<uint32_t>(e + 127) << 23);
}
// x 2^e for any e of a float's range, in two steps
__device__ __forceinline__ float times_pow2(float x, int e) {
  return x * pow2(e / 2) * pow2(e - e / 2);
}

__device__ __forceinline__ void mma_from(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2,
                                         uint32_t a3, uint32_t b0, uint32_t b1, float c0,
                                         float c1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
      "{%8,%9}, {%10,%11,%10,%11};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(c0), "f"(c1));
}

template <int N>
__device__ __forceinline__ void ldg_words(const uint8_t* p, uint32_t (&r)[N]) {
  if constexpr (N == 1)
    asm volatile("ld.global.L1::no_allocate.b32 %0, [%1];" : "=r"(r[0]) : "l"(p));
  else
    ldg(p, r);
}

// Sixteen keys' rows of a 4-bit page, as thread (r = lane / 4, q = lane % 4) needs them.
template <int D>
struct Rows4 {
  static constexpr int GR = D / 32;
  uint32_t k[2][GR];       // keys r and r + 8: 8 codes of each group
  uint32_t sk[2][GR / 2];  // their scales
  uint32_t v[4][GR / 2];   // keys 2q, 2q + 1, 2q + 8, 2q + 9: 4 codes of each group
  uint32_t sv[2][GR];      // their scales, two keys' each

  // codes: the first key's row of K; scales: its scales; v_after: from K to V
  __device__ __forceinline__ void load_k(const uint8_t* codes, const uint8_t* scales) {
    const int lane = threadIdx.x & 31, r = lane >> 2, q = lane & 3;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      ldg_words(codes + (r + 8 * x) * (D / 2) + q * (D / 8), k[x]);
      ldg_words(scales + (r + 8 * x) * (D / 16), sk[x]);
    }
  }
  __device__ __forceinline__ void load_v(const uint8_t* codes, const uint8_t* scales) {
    const int lane = threadIdx.x & 31, r = lane >> 2, q = lane & 3;
#pragma unroll
    for (int x = 0; x < 4; ++x)
      ldg_words(codes + (2 * q + (x & 1) + 8 * (x >> 1)) * (D / 2) + r * (D / 16), v[x]);
#pragma unroll
    for (int x = 0; x < 2; ++x) ldg_words(scales + (2 * q + 8 * x) * (D / 16), sv[x]);
  }
  // keys at or past n: what lies there may be anything, and 0 times NaN is NaN
  __device__ __forceinline__ void clear_from(int n) {
    const int q = threadIdx.x & 3;
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int y = 0; y < 2; ++y)
        if (2 * q + y + 8 * x >= n)
#pragma unroll
          for (int i = 0; i < GR / 2; ++i) sv[x][y * (GR / 2) + i] = 0;
  }
};

template <int D, int NT>
struct Keys4 {
  static constexpr int GR = D / 32;
  float o[NT][D / 16][4];     // tile (g, t): columns 32 g + 4 r + 2 t (+ 1: rows r + 8)
  float m[NT][2], l[NT][2];
  uint32_t q[NT][D / 16][2];  // Q^T: columns 32 g + 8 q ... + 7, the last four over 16
  float off[NT][GR][2];       // -8 2^-133 sum q of a group
  float back[NT][2];          // what undoes the column's power of two
  bool first;

  __device__ __forceinline__ void reset() {
    first = true;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      m[t][0] = m[t][1] = -INFINITY;
      l[t][0] = l[t][1] = 0.f;
#pragma unroll
      for (int i = 0; i < D / 16; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[t][i][e] = 0.f;
    }
  }

  __device__ __forceinline__ void load_q(const __nv_bfloat16* q_g, const DecGeom& geo) {
    constexpr uint32_t all = 0xffffffffu;
    const int lane = threadIdx.x & 31, r = lane >> 2, c = lane & 3;
    const int cols = geo.G * geo.tokens;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int h = 8 * t + r;
      uint4 w[GR];
      uint32_t top = 0;
#pragma unroll
      for (int g = 0; g < GR; ++g) {
        w[g] = make_uint4(0, 0, 0, 0);
        if (h < cols) {
          const int64_t row = (h >> geo.g_shift) * geo.Hq + (h & (geo.G - 1));
          w[g] = ld_plain(reinterpret_cast<const uint4*>(q_g + row * D) + 4 * g + c);
        }
        top = max(top, q4::abs_max8(w[g]));
      }
      top = max(top, __shfl_xor_sync(all, top, 1));
      top = max(top, __shfl_xor_sync(all, top, 2));
      // (a column of zeros, or with a NaN or infinity, stays as it is)
      const int e = top == 0 || top >= 0x7f80u ? 0 : kQTop + 127 - static_cast<int>(top >> 7);
      float sum[GR];
#pragma unroll
      for (int g = 0; g < GR; ++g) {
        const uint32_t x[4] = {w[g].x, w[g].y, w[g].z, w[g].w};
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float a = times_pow2(__uint_as_float(x[i] << 16), e);
          const float b = times_pow2(__uint_as_float(x[i] & 0xffff0000u), e);
          s += a + b;
          q[t][2 * g + i / 2][i & 1] = i < 2 ? pack_bf16x2(a, b)
                                             : pack_bf16x2(a * 0.0625f, b * 0.0625f);
        }
        s += __shfl_xor_sync(all, s, 1);
        s += __shfl_xor_sync(all, s, 2);
        sum[g] = s * pow2(-65) * pow2(-65);
      }
      const float undo = times_pow2(1.f, 53 - e);
      // from the lanes of a column (r) to those of its scores (2 c, 2 c + 1)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int from = 4 * (2 * c + x);
        back[t][x] = __shfl_sync(all, undo, from);
#pragma unroll
        for (int g = 0; g < GR; ++g) off[t][g][x] = -__shfl_sync(all, sum[g], from);
      }
    }
  }

  // S^T of a group of keys, times 2^(e - 133)
  __device__ __forceinline__ void scores(const Rows4<D>& f, float (&s)[NT][4]) const {
#pragma unroll
    for (int g = 0; g < GR; ++g) {
      const uint32_t x = f.k[0][g], y = f.k[1][g], x8 = x >> 8, y8 = y >> 8;
      const float s0 = __uint_as_float(g & 1 ? f.sk[0][g / 2] & 0xffff0000u : f.sk[0][g / 2] << 16);
      const float s1 = __uint_as_float(g & 1 ? f.sk[1][g / 2] & 0xffff0000u : f.sk[1][g / 2] << 16);
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        float c[4];
        mma_from(c, x & kLowNibbles, y & kLowNibbles, x8 & kLowNibbles, y8 & kLowNibbles,
                 q[t][2 * g][0], q[t][2 * g][1], off[t][g][0], off[t][g][1]);
        mma(c, x & kHighNibbles, y & kHighNibbles, x8 & kHighNibbles, y8 & kHighNibbles,
            q[t][2 * g + 1][0], q[t][2 * g + 1][1]);
        if (g == 0) {
          s[t][0] = c[0] * s0, s[t][1] = c[1] * s0;
          s[t][2] = c[2] * s1, s[t][3] = c[3] * s1;
        } else {
          s[t][0] = fmaf(c[0], s0, s[t][0]), s[t][1] = fmaf(c[1], s0, s[t][1]);
          s[t][2] = fmaf(c[2], s1, s[t][2]), s[t][3] = fmaf(c[3], s1, s[t][3]);
        }
      }
    }
  }

  // The same of rows of a 16-bit page.
  __device__ __forceinline__ void scores16(const uint8_t* kp, float (&s)[NT][4]) const {
    const int lane = threadIdx.x & 31, r = lane >> 2, c = lane & 3;
    float a[NT][4], b[NT][4];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) a[t][e] = b[t][e] = 0.f;
#pragma unroll
    for (int g = 0; g < GR; ++g) {
      uint32_t x[4], y[4];
      ldg(kp + (r * D + 32 * g + 8 * c) * 2, x);
      ldg(kp + ((r + 8) * D + 32 * g + 8 * c) * 2, y);
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        mma(a[t], x[0], y[0], x[1], y[1], q[t][2 * g][0], q[t][2 * g][1]);
        mma(b[t], x[2], y[2], x[3], y[3], q[t][2 * g + 1][0], q[t][2 * g + 1][1]);
      }
    }
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        s[t][e] = fmaf(b[t][e], 16.f, a[t][e]) * pow2(-66) * pow2(-67);
  }

  // scores -> P^T (B operand of the V product), times 2^kPBias; the column of token i of
  // the request's last `tokens` sees the keys below n - (tokens - 1 - i)
  __device__ __forceinline__ void softmax(float (&s)[NT][4], int n, const DecGeom& geo,
                                          uint32_t (&p)[NT][2]) {
    const int lane = threadIdx.x & 31, r = lane >> 2;
    const float scale = geo.scale_log2 * pow2(80);
    bool grow = false;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const float f = back[t][x];
        s[t][x] *= scale, s[t][x] *= f;
        s[t][x + 2] *= scale, s[t][x + 2] *= f;
      }
    if (n < kGroup + geo.tokens - 1) {
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int token = (8 * t + 2 * (lane & 3) + (e & 1)) >> geo.g_shift;
          if (r + 8 * (e >> 1) + geo.tokens - 1 - token >= n) s[t][e] = -INFINITY;
        }
    }
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) grow |= s[t][e] - m[t][e & 1] > kRaise4;
    if (first || __any_sync(0xffffffffu, grow)) {
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          float mx = fmaxf(s[t][x], s[t][x + 2]);
#pragma unroll
          for (int d = 4; d < 32; d <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
          if (first) {
            m[t][x] = mx;
          } else if (mx > m[t][x]) {
            const float alpha = ex2_approx(m[t][x] - mx);
            l[t][x] *= alpha;
#pragma unroll
            for (int i = 0; i < D / 16; ++i) {
              o[t][i][x] *= alpha;
              o[t][i][x + 2] *= alpha;
            }
            m[t][x] = mx;
          }
        }
      first = false;
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      float e[4];
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        // (a column may have no key yet: its maximum is -inf then)
        e[x] = s[t][x] == -INFINITY ? 0.f : ex2_approx(s[t][x] - m[t][x & 1] + kPBias);
        l[t][x & 1] += e[x];
      }
      p[t][0] = transpose8(pack_bf16x2(e[0], e[1]));
      p[t][1] = transpose8(pack_bf16x2(e[2], e[3]));
    }
  }

  // O^T += V^T P^T
  __device__ __forceinline__ void values(const Rows4<D>& f, const uint32_t (&p)[NT][2]) {
#pragma unroll
    for (int g = 0; g < GR; ++g) {
      const uint32_t half = g & 1 ? 0x7632 : 0x5410;
      const uint32_t x = __byte_perm(f.v[0][g / 2], f.v[1][g / 2], half), x8 = x >> 8;
      const uint32_t y = __byte_perm(f.v[2][g / 2], f.v[3][g / 2], half), y8 = y >> 8;
      const uint32_t s0 = __byte_perm(f.sv[0][g / 2], f.sv[0][g / 2 + GR / 2], half);
      const uint32_t s1 = __byte_perm(f.sv[1][g / 2], f.sv[1][g / 2 + GR / 2], half);
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const uint32_t b0 = q4::mul_bf16x2(p[t][0], s0), b1 = q4::mul_bf16x2(p[t][1], s1);
        mma(o[t][2 * g], x & kLowNibbles, x & kHighNibbles, y & kLowNibbles, y & kHighNibbles, b0,
            b1);
        mma(o[t][2 * g + 1], x8 & kLowNibbles, x8 & kHighNibbles, y8 & kLowNibbles,
            y8 & kHighNibbles, b0, b1);
        // -8 and -128 times 2^-133
        mma(o[t][2 * g], 0x80088008u, 0x80808080u, 0x80088008u, 0x80808080u, b0, b1);
        mma(o[t][2 * g + 1], 0x80088008u, 0x80808080u, 0x80088008u, 0x80808080u, b0, b1);
      }
    }
  }

  // The same of rows of a 16-bit page, keys at or past n left out.
  __device__ __forceinline__ void values16(const uint8_t* vp, int n, const uint32_t (&p)[NT][2]) {
    const int lane = threadIdx.x & 31, r = lane >> 2, c = lane & 3;
    uint32_t b[NT][2], b16[NT][2];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        // P 2^-133, and 16 times that for the rows r + 8
        b[t][i] = q4::mul_bf16x2(q4::mul_bf16x2(p[t][i], 0x1e801e80u), 0x1e001e00u);
        b16[t][i] = q4::mul_bf16x2(b[t][i], 0x41804180u);
      }
#pragma unroll
    for (int g = 0; g < GR; ++g) {
      uint32_t v[4][2];
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const int key = 2 * c + (x & 1) + 8 * (x >> 1);
        v[x][0] = v[x][1] = 0;
        if (key < n) ldg(vp + (key * D + 32 * g + 4 * r) * 2, v[x]);
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t a0 = __byte_perm(v[0][i], v[1][i], 0x5410);
        const uint32_t a1 = __byte_perm(v[0][i], v[1][i], 0x7632);
        const uint32_t a2 = __byte_perm(v[2][i], v[3][i], 0x5410);
        const uint32_t a3 = __byte_perm(v[2][i], v[3][i], 0x7632);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          mma(o[t][2 * g + i], a0, 0, a2, 0, b[t][0], b[t][1]);
          mma(o[t][2 * g + i], 0, a1, 0, a3, b16[t][0], b16[t][1]);
        }
      }
    }
  }

  // The groups first, first + every, ... of piece w of a request of T keys, to O, reference
  // maxima and sums as decode_cta merges them.
  __device__ __forceinline__ void run(const DecGeom& geo, const DecPiece& w, int T, int first_group,
                                      int every, const __nv_bfloat16* q_g, const uint8_t* pool_k,
                                      int64_t plane16, const int32_t* block_table,
                                      int32_t* status) {
    const int lane = threadIdx.x & 31;
    const uint32_t k1 = static_cast<uint32_t>(w.k1), mask = static_cast<uint32_t>(geo.ps - 1);
    const uint64_t head = q4_head_bytes(D, geo.ps);
    const int64_t plane4 = static_cast<int64_t>(geo.q4_pages) * geo.Hkv * head;
    const uint8_t* q4_k = geo.q4_cache + geo.layer * 2 * plane4;
    auto key_of = [&](int i) {
      return static_cast<uint32_t>(w.k0) + static_cast<uint32_t>(first_group + i * every) * kGroup;
    };
    // lane i looks up the warp's groups i, i + 32, ...: the address of the first key's row,
    // lowest bit set in a 16-bit page, 0: none (bad, or past the piece)
    auto look = [&](uint32_t key) -> uint64_t {
      if (key >= k1) return 0;
      const int64_t e = static_cast<int64_t>(w.b) * geo.max_blocks + (key >> geo.ps_shift);
      const int p4 = ld_plain(geo.q4_table + e);
      const uint32_t slot = key & mask;
      if (p4 >= 0) {
        if (p4 < geo.q4_pages)
          return reinterpret_cast<uint64_t>(
              q4_k + (static_cast<uint64_t>(p4) * geo.Hkv + w.g) * head + slot * (D / 2));
      } else {
        const int page = ld_plain(block_table + e);
        if (page >= 0 && page < geo.num_pages)
          return reinterpret_cast<uint64_t>(
                     pool_k + ((static_cast<int64_t>(page) * geo.Hkv + w.g) * geo.ps + slot) * D * 2) |
                 1;
      }
      record_error(status, GC_ERR_OUT_OF_RANGE);
      return 0;
    };
    uint64_t cur = look(key_of(lane));
    reset();
    load_q(q_g, geo);
    uint64_t nxt = key_of(32) < k1 ? look(key_of(32 + lane)) : 0;
    Rows4<D> f[2];
    uint64_t at[2];
    // Two groups are under way: one is loaded as soon as the one before the last is done.
    auto fetch = [&](int i, Rows4<D>& to) -> uint64_t {
      if (key_of(i) >= k1) return 0;
      if ((i & 31) == 0 && i > 0) {
        cur = nxt;
        nxt = key_of(i + 32) < k1 ? look(key_of(i + 32 + lane)) : 0;
      }
      const uint64_t a = __shfl_sync(0xffffffffu, cur, i & 31);
      if (a != 0 && !(a & 1)) {
        const uint8_t* codes = reinterpret_cast<const uint8_t*>(a);
        const uint32_t slot = key_of(i) & mask;
        const uint8_t* scales = codes + (geo.ps * 8 - static_cast<int>(slot) * 7) * (D / 16);
        to.load_k(codes, scales);
        to.load_v(codes + plane4, scales + plane4);
      }
      return a;
    };
    at[0] = fetch(0, f[0]);
    at[1] = fetch(1, f[1]);
    for (int i = 0; key_of(i) < k1; i += 2) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        if (key_of(i + u) >= k1) break;
        const uint64_t a = at[u];
        // keys of the group before the request's end (16 or more: all of them)
        const int n = T - static_cast<int>(key_of(i + u));
        float s[NT][4];
        uint32_t p[NT][2];
        if (a != 0 && !(a & 1)) {
          scores(f[u], s);
          softmax(s, n, geo, p);
          if (n < kGroup) f[u].clear_from(n);
          values(f[u], p);
        } else if (a != 0) {
          const uint8_t* kp = reinterpret_cast<const uint8_t*>(a & ~1ull);
          scores16(kp, s);
          softmax(s, n, geo, p);
          values16(kp + plane16, n, p);
        }
        at[u] = fetch(i + u + 2, f[u]);
      }
    }
    // the powers of two leave: 2^(kPBias - 133) of O, 16 of its rows r + 8, 2^kPBias of l
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      l[t][0] *= pow2(-90), l[t][1] *= pow2(-90);
#pragma unroll
      for (int i = 0; i < D / 16; ++i) {
        o[t][i][0] *= pow2(43), o[t][i][1] *= pow2(43);
        o[t][i][2] *= pow2(39), o[t][i][3] *= pow2(39);
      }
    }
  }
};

}  // namespace dec
}  // namespace
}  // namespace gc

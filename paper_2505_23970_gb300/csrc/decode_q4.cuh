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
//  * the offset 8 is one more product: for S of a key's scales with the groups' sums of
//    -8 q, in three bf16 parts that make up their 24 bits, for O of a constant with P;
//  * S is scaled group by group in binary32, S += s_g D_g; P is scaled by V's s_g before
//    its product and P s_g rounded once to bf16, at most 2^-8 of a term.  (Rounding P alone,
//    and scaling it after the transposition, is a rounding more for 30 instructions less of
//    299 a group of keys: error against 64 bits 0.0026 instead of 0.0022, the output's own
//    rounding being 0.0017.)
// Powers of two keep everything in range: Q's columns are brought to 2^100 at the most, P
// is 2^90 2^(x - m), and both leave again exactly.
//
// Keys and scales come through shared memory, copied asynchronously a pair of groups ahead
// (a probe of nothing but copies: random pieces of 1152 bytes 6.9 TB/s so, 5.7 by loads to
// registers, of which there are too few for a group more; this kernel without its products
// copies 5.4 TB/s, and why not more is not known).  Codes as e4m3 with m16n8k32 products would save half of K's
// masks, but that product is not native here (it is carried out as conversions and f16
// products): 32 documents 366 us instead of 224.
#pragma once

#include "decode_mma.cuh"
#include "q4_format.cuh"

namespace gc {

// A call's sizes and where its keys are.
struct Dec4Geom {
  int32_t batch, Hq, Hkv, G, g_shift, tokens, ps, ps_shift, num_pages, q4_pages, max_blocks;
  int32_t unit_shift;  // keys per unit of work, log2 (at least 5)
  float scale_log2;
  uint32_t q4_page;     // bytes of a 4-bit page's plane
  int64_t q4_plane;     // of all of them
  int64_t plane16;      // bytes of the pool's plane
  const uint8_t* q4_k;  // the layer's K
  const uint8_t* pool_k;
  const int32_t* q4_table;
  const int32_t* block_table;
};

namespace {
namespace dec {

constexpr int kQTop = 100;         // exponent of a column's largest |q|
constexpr float kPBias = 90.0f;    // P is 2^kPBias at the reference maximum
constexpr float kRaise4 = 8.0f;    // scores this far above it raise it
constexpr float kNone = -3e38f;    // the reference maximum of a column without a key yet
constexpr uint32_t kLowNibbles = 0x000f000fu, kHighNibbles = 0x00f000f0u;

__device__ __forceinline__ float pow2(int e) {  // -126 <= e <= 127
  return __uint_as_float(static_cast<uint32_t>(e + 127) << 23);
}
// x 2^e for any e of a float's range, in two steps
__device__ __forceinline__ float times_pow2(float x, int e) {
  return x * pow2(e / 2) * pow2(e - e / 2);
}

// x to 8 bits, towards 0
__device__ __forceinline__ float bf16_part(float x) {
  return __uint_as_float(__float_as_uint(x) & 0xffff0000u);
}

__device__ __forceinline__ void mma_first(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2,
                                          uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
      "{%8,%9}, {%10,%10,%10,%10};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}

// A group of keys in shared memory: K's codes and scales, V's codes and scales.
template <int D>
struct Stage4 {
  static constexpr int GR = D / 32;
  static constexpr int kCodes = kGroup * D / 2, kScales = kGroup * D / 16;
  static constexpr int kBytes = 2 * (kCodes + kScales);
};

// (a predicate in place of a branch: branches are most of what a small loop adds)
__device__ __forceinline__ void copy16_if(bool on, uint32_t to, const uint8_t* from) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %2, 0;\n\t"
               "@p cp.async.cg.shared.global [%0], [%1], 16;\n\t}" ::"r"(to),
               "l"(from), "r"(static_cast<uint32_t>(on))
               : "memory");
}
// Keeps a value in its register: worked out again at each use it would take more
// instructions than all else that the use is about.
__device__ __forceinline__ uint32_t kept(uint32_t x) {
  asm volatile("" : "+r"(x));
  return x;
}

// What a lane copies of a group of keys, and where it reads its operands in a stage.  Row i
// of S^T and of P^T is the key i & 8 + 4 (i & 1) + (i & 7) / 2: with this order the rows of V
// that the lanes of a warp read together lie side by side.
template <int D>
struct Parts4 {
  static constexpr int kCodes = Stage4<D>::kCodes, kScales = Stage4<D>::kScales;
  uint32_t k, s, v;  // codes of its K rows, their (and V's) scales, codes of its V rows
  uint32_t bytes;

  __device__ __forceinline__ static int row() {  // the key of its first row of P
    const int r = (threadIdx.x & 31) >> 2;
    return (r & 1) * 4 + (r >> 1);
  }
  __device__ __forceinline__ Parts4() {
    const int lane = threadIdx.x & 31, r = lane >> 2, c = lane & 3;
    k = kept(row() * (D / 2) + c * (D / 8));
    s = kept(kCodes + row() * (D / 16));
    v = kept(kCodes + kScales + c * (D / 2) + r * (D / 16));
    bytes = kept(16 * lane);
  }
  // codes: the row of K of the group's first key; after: from there to its scales; plane:
  // from K to V
  __device__ __forceinline__ void copy_if(bool on, uint32_t to, const uint8_t* codes, int after,
                                          int64_t plane) const {
    constexpr int kV = kCodes + kScales;
    codes += bytes;
    to += bytes;
    const uint8_t* const v = codes + plane;
#pragma unroll
    for (int i = 0; i < kCodes / 512; ++i) {
      copy16_if(on, to + 512 * i, codes + 512 * i);
      copy16_if(on, to + kV + 512 * i, v + 512 * i);
    }
    const bool scales = on && bytes < kScales;
    copy16_if(scales, to + kCodes, codes + after);
    copy16_if(scales, to + kV + kCodes, v + after);
  }
};

// (C++ loads, which the compiler may move between the barriers of the loop)
template <int N>
__device__ __forceinline__ void lds_words(const uint8_t* at, uint32_t (&r)[N]) {
  static_assert(N == 1 || N == 2 || N == 4, "a load");
  if constexpr (N == 1) {
    r[0] = *reinterpret_cast<const uint32_t*>(at);
  } else if constexpr (N == 2) {
    const uint2 v = *reinterpret_cast<const uint2*>(at);
    r[0] = v.x, r[1] = v.y;
  } else {
    const uint4 v = *reinterpret_cast<const uint4*>(at);
    r[0] = v.x, r[1] = v.y, r[2] = v.z, r[3] = v.w;
  }
}
__device__ __forceinline__ float half_f32(uint32_t pair, int i) {  // of two bf16
  return __uint_as_float(i ? pair & 0xffff0000u : pair << 16);
}

template <int D, int NT>
struct Keys4 {
  static constexpr int GR = D / 32;
  float o[NT][D / 16][4];     // tile (g, t): columns 32 g + 4 r + 2 t (+ 1: rows r + 8)
  float m[NT][2], l[NT][2];
  uint32_t q[NT][D / 16][2];  // Q^T: columns 32 g + 8 c ... + 7, the last four over 16
  uint32_t off[NT][GR / 2];   // -8 2^-133 times the groups' sums of q (B operand, see set_q)
  float scale[NT][2];         // softmax_scale log2(e), and what undoes the powers of two

  __device__ __forceinline__ void reset() {
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      m[t][0] = m[t][1] = kNone;
      l[t][0] = l[t][1] = 0.f;
#pragma unroll
      for (int i = 0; i < D / 16; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[t][i][e] = 0.f;
    }
  }

  // The columns as they are: 32 g + 8 c ... + 7 of column 8 t + r.
  __device__ __forceinline__ void load_q(const __nv_bfloat16* q_g, const Dec4Geom& geo,
                                         uint4 (&w)[NT][GR]) {
    const int lane = threadIdx.x & 31, r = lane >> 2, c = lane & 3;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int h = 8 * t + r;
      const int64_t row = (h >> geo.g_shift) * geo.Hq + (h & (geo.G - 1));
#pragma unroll
      for (int g = 0; g < GR; ++g) {
        w[t][g] = make_uint4(0, 0, 0, 0);
        if (h < geo.G * geo.tokens)
          w[t][g] = ld_plain(reinterpret_cast<const uint4*>(q_g + row * D) + 4 * g + c);
      }
    }
  }
  __device__ __forceinline__ void set_q(const uint4 (&all_w)[NT][GR], const Dec4Geom& geo) {
    constexpr uint32_t all = 0xffffffffu;
    const int c = threadIdx.x & 3;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const uint4(&w)[GR] = all_w[t];
      uint32_t top = 0;
#pragma unroll
      for (int g = 0; g < GR; ++g) top = max(top, q4::abs_max8(w[g]));
      top = max(top, __shfl_xor_sync(all, top, 1));
      top = max(top, __shfl_xor_sync(all, top, 2));
      // (a column of zeros, or with a NaN or infinity, stays as it is; 20 keeps the scale
      // in range where |q| passes 2^80)
      const int e = top == 0 || top >= 0x7f80u
                        ? kQTop
                        : max(20, kQTop + 127 - static_cast<int>(top >> 7));
      float sum[GR];
#pragma unroll
      for (int g = 0; g < GR; ++g) {
        const uint32_t x[4] = {w[g].x, w[g].y, w[g].z, w[g].w};
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float a = times_pow2(half_f32(x[i], 0), e);
          const float b = times_pow2(half_f32(x[i], 1), e);
          s += a + b;
          q[t][2 * g + i / 2][i & 1] = i < 2 ? pack_bf16x2(a, b)
                                             : pack_bf16x2(a * 0.0625f, b * 0.0625f);
        }
        s += __shfl_xor_sync(all, s, 1);
        s += __shfl_xor_sync(all, s, 2);
        sum[g] = s * -pow2(-65) * pow2(-65);
      }
      // Row k of the operand is part k / GR of group k % GR's sum: two rows (groups) to a
      // register, parts 0 to 2 in turn; a key's scales are the other operand as they lie.
#pragma unroll
      for (int i = 0; i < GR / 2; ++i) {
        const int k = 2 * c + 8 * i, part = k / GR;
        float v[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          float s = sum[j];
          if (GR == 4 && k % GR) s = sum[GR - 2 + j];
          const float hi = bf16_part(s), mid = bf16_part(s - hi);
          v[j] = part == 0 ? hi : part == 1 ? mid : part == 2 ? s - hi - mid : 0.f;
        }
        off[t][i] = pack_bf16x2(v[0], v[1]);
      }
      // (never 0, which times the -infinity of a masked score would be NaN)
      const float undo = fmaxf(times_pow2(geo.scale_log2, 133 - e), pow2(-126));
      // from the lanes of a column (r) to those of its scores (2 c, 2 c + 1)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int from = 4 * (2 * c + x);
        scale[t][x] = __shfl_sync(all, undo, from);
      }
    }
  }

  // S^T of a group of keys, times 2^(e - 133)
  __device__ __forceinline__ void scores(const uint8_t* at, const Parts4<D>& mine,
                                         float (&s)[NT][4]) const {
    uint32_t k[2][GR], sk[2][GR / 2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      lds_words(at + mine.k + 8 * x * (D / 2), k[x]);
      lds_words(at + mine.s + 8 * x * (D / 16), sk[x]);
    }
    // -8 2^-133 sum_g s_g sum q
    const bool odd = GR == 4 && (mine.bytes & 16);
    const uint32_t x01 = odd ? sk[0][GR / 2 - 1] : sk[0][0];
    const uint32_t y01 = odd ? sk[1][GR / 2 - 1] : sk[1][0];
#pragma unroll
    for (int t = 0; t < NT; ++t)
      mma_first(s[t], x01, y01, GR == 4 ? x01 : 0u, GR == 4 ? y01 : 0u, off[t][0],
                GR == 4 ? off[t][GR / 2 - 1] : 0u);
#pragma unroll
    for (int g = 0; g < GR; ++g) {
      const uint32_t x = k[0][g], y = k[1][g], x8 = x >> 8, y8 = y >> 8;
      const float s0 = half_f32(sk[0][g / 2], g & 1), s1 = half_f32(sk[1][g / 2], g & 1);
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        float d[4];
        mma_first(d, x & kLowNibbles, y & kLowNibbles, x8 & kLowNibbles, y8 & kLowNibbles,
                  q[t][2 * g][0], q[t][2 * g][1]);
        mma(d, x & kHighNibbles, y & kHighNibbles, x8 & kHighNibbles, y8 & kHighNibbles,
            q[t][2 * g + 1][0], q[t][2 * g + 1][1]);
        s[t][0] = fmaf(d[0], s0, s[t][0]), s[t][1] = fmaf(d[1], s0, s[t][1]);
        s[t][2] = fmaf(d[2], s1, s[t][2]), s[t][3] = fmaf(d[3], s1, s[t][3]);
      }
    }
  }

  // The same of rows of a 16-bit page, which are taken times 2^-60 so that no product with
  // Q's columns overflows.
  __device__ __forceinline__ void scores16(const uint8_t* kp, const Parts4<D>& mine,
                                           float (&s)[NT][4]) const {
    const int c = threadIdx.x & 3;
    float a[NT][4], b[NT][4];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) a[t][e] = b[t][e] = 0.f;
#pragma unroll
    for (int g = 0; g < GR; ++g) {
      uint32_t x[4], y[4];
      ldg(kp + (mine.row() * D + 32 * g + 8 * c) * 2, x);
      ldg(kp + ((mine.row() + 8) * D + 32 * g + 8 * c) * 2, y);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[i] = q4::mul_bf16x2(x[i], 0x21802180u);
        y[i] = q4::mul_bf16x2(y[i], 0x21802180u);
      }
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        mma(a[t], x[0], y[0], x[1], y[1], q[t][2 * g][0], q[t][2 * g][1]);
        mma(b[t], x[2], y[2], x[3], y[3], q[t][2 * g + 1][0], q[t][2 * g + 1][1]);
      }
    }
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[t][e] = fmaf(b[t][e], 16.f, a[t][e]) * pow2(-73);
  }

  // The token of the request's last `tokens` that column 2 c + x of tile t is of: token i sees
  // the keys below n - (tokens - 1) + i.
  __device__ __forceinline__ static int token(int t, int x, const Dec4Geom& geo) {
    return (8 * t + 2 * static_cast<int>(threadIdx.x & 3) + x) >> geo.g_shift;
  }
  __device__ __forceinline__ void mask(float (&s)[NT][4], const Parts4<D>& mine, int n,
                                       const Dec4Geom& geo) const {
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (mine.row() + 8 * (e >> 1) + geo.tokens - 1 - token(t, e & 1, geo) >= n)
          s[t][e] = -INFINITY;
  }

  // scores of H groups -> P, times 2^kPBias
  template <int H>
  __device__ __forceinline__ void softmax(float (&s)[H][NT][4]) {
    float top = -INFINITY;
    float x[H][NT][4];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const float b[2] = {kPBias - m[t][0], kPBias - m[t][1]};
#pragma unroll
      for (int h = 0; h < H; ++h)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x[h][t][e] = fmaf(s[h][t][e], scale[t][e & 1], b[e & 1]);
          top = fmaxf(top, x[h][t][e]);
        }
    }
    if (__any_sync(0xffffffffu, top > kPBias + kRaise4)) {
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float mx = -INFINITY;
#pragma unroll
          for (int h = 0; h < H; ++h) mx = fmaxf(mx, fmaxf(s[h][t][i], s[h][t][i + 2]));
          mx *= scale[t][i];
#pragma unroll
          for (int d = 4; d < 32; d <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
          if (mx > m[t][i]) {
            const float alpha = ex2_approx(m[t][i] - mx);
            l[t][i] *= alpha;
#pragma unroll
            for (int j = 0; j < D / 16; ++j) {
              o[t][j][i] *= alpha;
              o[t][j][i + 2] *= alpha;
            }
            m[t][i] = mx;
          }
#pragma unroll
          for (int h = 0; h < H; ++h) {
            x[h][t][i] = fmaf(s[h][t][i], scale[t][i], kPBias - m[t][i]);
            x[h][t][i + 2] = fmaf(s[h][t][i + 2], scale[t][i], kPBias - m[t][i]);
          }
        }
    }
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s[h][t][e] = ex2_approx(x[h][t][e]);
          l[t][e & 1] += s[h][t][e];
        }
  }

  // O^T += V^T P^T; kTail: a P of 0, that of a column that does not see the key, adds nothing
  // whatever the key's scale is (0 times a NaN or an infinity would).  (That holds for keys at
  // or past n too; clearing their scales as they are read besides saves 12 bytes of spills:
  // 64 multi-turn contexts 68.5 us, without it 69.5.)
  template <bool kTail>
  __device__ __forceinline__ void values(const uint8_t* at, const Parts4<D>& mine, int n,
                                         const float (&p)[NT][4]) {
    uint32_t v[4][GR / 2], sv[2][GR / 2];
#pragma unroll
    for (int x = 0; x < 4; ++x) lds_words(at + mine.v + 4 * x * (D / 2), v[x]);
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      lds_words(at + mine.s + Stage4<D>::kCodes + Stage4<D>::kScales + 8 * x * (D / 16), sv[x]);
      if (kTail && mine.row() + 8 * x >= n)
#pragma unroll
        for (int i = 0; i < GR / 2; ++i) sv[x][i] = 0;
    }
#pragma unroll
    for (int g = 0; g < GR; ++g) {
      const uint32_t half = g & 1 ? 0x7632 : 0x5410;
      const uint32_t x = __byte_perm(v[0][g / 2], v[1][g / 2], half), x8 = x >> 8;
      const uint32_t y = __byte_perm(v[2][g / 2], v[3][g / 2], half), y8 = y >> 8;
      const float s0 = half_f32(sv[0][g / 2], g & 1), s1 = half_f32(sv[1][g / 2], g & 1);
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        float ps[4] = {p[t][0] * s0, p[t][1] * s0, p[t][2] * s1, p[t][3] * s1};
        if constexpr (kTail)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (p[t][e] == 0.f) ps[e] = 0.f;
        const uint32_t b0 = transpose8(pack_bf16x2(ps[0], ps[1]));
        const uint32_t b1 = transpose8(pack_bf16x2(ps[2], ps[3]));
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

  // The same of rows of a 16-bit page.  Keys that some column does not see are added one by
  // one where they are seen: what a page holds may be infinite, and 0 times that is NaN.
  __device__ __forceinline__ void values16(const uint8_t* vp, int n, const float (&p)[NT][4],
                                           const Dec4Geom& geo) {
    const int lane = threadIdx.x & 31, r = lane >> 2, c = lane & 3;
    const int by_all = n - (geo.tokens - 1);
    uint32_t b[NT][2], b16[NT][2];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        // P 2^-133, and 16 times that for the rows r + 8
        b[t][i] = transpose8(pack_bf16x2(p[t][2 * i], p[t][2 * i + 1]));
        b[t][i] = q4::mul_bf16x2(q4::mul_bf16x2(b[t][i], 0x1e801e80u), 0x1e001e00u);
        b16[t][i] = q4::mul_bf16x2(b[t][i], 0x41804180u);
      }
#pragma unroll
    for (int g = 0; g < GR; ++g) {
      uint32_t v[4][2];
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const int key = c + 4 * x;
        v[x][0] = v[x][1] = 0;
        if (key < by_all) ldg(vp + (key * D + 32 * g + 4 * r) * 2, v[x]);
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
#pragma unroll 1
    for (int key = max(by_all, 0); key < min(n, kGroup); ++key) {
      const int from = ((key & 3) * 2 + (key >> 2 & 1)) * 4 + c;  // the lane with its P
      float w[NT][2];
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int x = 0; x < 2; ++x)
          w[t][x] = __shfl_sync(0xffffffffu, key < 8 ? p[t][x] : p[t][x + 2], from) * pow2(-65) *
                    pow2(-68);
#pragma unroll
      for (int g = 0; g < GR; ++g) {
        uint32_t v[2];
        ldg(vp + (key * D + 32 * g + 4 * r) * 2, v);
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            if (key >= by_all + token(t, x, geo)) continue;
            const float y = w[t][x], y16 = 16.f * y;
            o[t][2 * g][x] = fmaf(y, half_f32(v[0], 0), o[t][2 * g][x]);
            o[t][2 * g][x + 2] = fmaf(y16, half_f32(v[0], 1), o[t][2 * g][x + 2]);
            o[t][2 * g + 1][x] = fmaf(y, half_f32(v[1], 0), o[t][2 * g + 1][x]);
            o[t][2 * g + 1][x + 2] = fmaf(y16, half_f32(v[1], 1), o[t][2 * g + 1][x + 2]);
          }
      }
    }
  }

  // Any group: in 16 bits, with keys that some column does not see, or none.
  template <typename Entry, typename WideRow>
  __device__ __forceinline__ void one(const uint8_t* from, uint32_t key, int h, uint32_t ready,
                                      int T, uint32_t k1, const Parts4<D>& mine,
                                      const Entry& entry, const WideRow& wide_row,
                                      const Dec4Geom& geo) {
    key += h * kGroup;
    from += h * Stage4<D>::kBytes;
    if (key >= k1) return;
    const bool four = ready >> h & 1;
    const uint8_t* kp = nullptr;
    if (!four) kp = wide_row(key, entry(key));
    if (!four && kp == nullptr) return;
    const int n = T - static_cast<int>(key);
    float s[1][NT][4];
    if (four)
      scores(from, mine, s[0]);
    else
      scores16(kp, mine, s[0]);
    mask(s[0], mine, n, geo);
    softmax(s);
    if (four)
      values<true>(from, mine, n, s[0]);
    else
      values16(kp + geo.plane16, n, s[0], geo);
  }

  // The keys of piece w of a request of T keys, two groups at a time, to O, reference
  // maxima and sums.  `ring`: the warp's kStages stages in shared memory, each for a pair.
  template <int kStages>
  __device__ __forceinline__ void run(const uint8_t* ring_at, const Dec4Geom& geo,
                                      const DecPiece& w, int T, const __nv_bfloat16* q_g,
                                      int32_t* status) {
    constexpr uint32_t kStage = 2 * Stage4<D>::kBytes, step = 2 * kGroup;
    const int lane = threadIdx.x & 31;
    // (unsigned: look-ups run past a piece that may end near 2^31)
    const uint32_t k1 = static_cast<uint32_t>(w.k1), slots = static_cast<uint32_t>(geo.ps - 1);
    const uint8_t* q4_k = geo.q4_k + static_cast<uint64_t>(w.g) * q4_head_bytes(D, geo.ps);
    auto entry_of = [&](uint32_t key) {
      return static_cast<int64_t>(w.b) * geo.max_blocks + (key >> geo.ps_shift);
    };
    // The row of K of a key that is in no 4-bit page, null: in a bad one.
    auto wide_row = [&](uint32_t key, int p4) -> const uint8_t* {
      const int page = p4 < 0 ? ld_plain(geo.block_table + entry_of(key)) : -1;
      if (page < 0 || page >= geo.num_pages) {
        record_error(status, GC_ERR_OUT_OF_RANGE);
        return nullptr;
      }
      return geo.pool_k +
             ((static_cast<int64_t>(page) * geo.Hkv + w.g) * geo.ps + (key & slots)) * D * 2;
    };
    // A key's entry of the 4-bit table, -1 past the piece.  Nothing is asked of it yet: a
    // window's entries are on their way while the window before is worked on.
    auto entry = [&](uint32_t key) {
      return key < k1 ? ld_plain(geo.q4_table + entry_of(key)) : -1;
    };
    auto in_4_bits = [&](int p4) { return p4 < geo.q4_pages ? p4 : -1; };
    // A window of 16 pairs is looked up at once, lane i a group of pair i / 2, and the next
    // one ahead of its use.
    const uint32_t key0 = static_cast<uint32_t>(w.k0);
    const uint32_t mine_in = static_cast<uint32_t>(lane) * kGroup;
    uint4 q_words[NT][GR];
    load_q(q_g, geo, q_words);
    int cur = entry(key0 + mine_in);
    const Parts4<D> mine;
    // Pairs are copied kStages - 1 before their turn, into the stage whose reader of the round
    // before is done in every lane.  Bits 2 j, 2 j + 1 of `ready`: the groups of pair j from
    // now on are in 4 bits.
    const uint32_t ring = static_cast<uint32_t>(__cvta_generic_to_shared(ring_at));
    const uint32_t end = ring + kStages * kStage;
    uint32_t to = ring, ahead = key0, ready = 0;
    int ahead_i = 0, nxt = -1;
    auto fetch = [&]() {
      ready >>= 2;
      if (ahead_i == 32) {
        ahead_i = 0;
        cur = in_4_bits(nxt);
        nxt = entry(ahead + 16 * step + mine_in);
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int page = __shfl_sync(0xffffffffu, cur, ahead_i + h);  // -1 past the piece
        const uint32_t slot = (ahead + h * kGroup) & slots;
        mine.copy_if(page >= 0, to + h * Stage4<D>::kBytes,
                     q4_k + (static_cast<uint64_t>(static_cast<uint32_t>(page)) * geo.q4_page +
                             slot * (D / 2)),
                     static_cast<int>(geo.ps * 8 - slot * 7) * (D / 16), geo.q4_plane);
        ready |= (static_cast<uint32_t>(~page) >> 31) << (2 * (kStages - 1) + h);
      }
      ahead += step;
      ahead_i += 2;
      to = to + kStage == end ? ring : to + kStage;
      asm volatile("cp.async.commit_group;" ::: "memory");
    };
    cur = in_4_bits(cur);
    for (int i = 0; i < kStages - 1; ++i) fetch();
    static_assert(kStages <= 16, "the first window has the first stages' pairs");
    nxt = entry(key0 + 16 * step + mine_in);
    reset();
    set_q(q_words, geo);
    uint32_t from = 0;
    // keys below this are seen by every column
    const uint32_t seen = min(k1, static_cast<uint32_t>(T - geo.tokens + 1));
    for (uint32_t key = key0; key < k1; key += step) {
      asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 2) : "memory");
      __syncwarp();
      fetch();
      // (the same in every lane; the vote says so)
      if (__all_sync(0xffffffffu, (ready & 3) == 3 && key + 2 * kGroup <= seen)) {
        float s[2][NT][4];
        const uint8_t* const at = ring_at + from;
        scores(at, mine, s[0]);
        scores(at + Stage4<D>::kBytes, mine, s[1]);
        softmax(s);
        values<false>(at, mine, kGroup, s[0]);
        values<false>(at + Stage4<D>::kBytes, mine, kGroup, s[1]);
      } else {
#pragma unroll 1
        for (int h = 0; h < 2; ++h)
          one(ring_at + from, key, h, ready, T, k1, mine, entry, wide_row, geo);
      }
      from = from + kStage == kStages * kStage ? 0 : from + kStage;
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    // the powers of two leave: 2^(kPBias - 133) of O, 16 of its rows r + 8, 2^kPBias of l
#pragma unroll
    for (int t = 0; t < NT; ++t) {
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        l[t][x] *= pow2(-90);
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) l[t][x] += __shfl_xor_sync(0xffffffffu, l[t][x], d);
      }
#pragma unroll
      for (int i = 0; i < D / 16; ++i) {
        o[t][i][0] *= pow2(43), o[t][i][1] *= pow2(43);
        o[t][i][2] *= pow2(39), o[t][i][3] *= pow2(39);
      }
    }
  }

  // Four columns 32 g + 4 r ... of the head of tile t, column 2 c + x.
  __device__ __forceinline__ float4 four(int t, int g, int x) const {
    return make_float4(o[t][2 * g][x], o[t][2 * g][x + 2], o[t][2 * g + 1][x],
                       o[t][2 * g + 1][x + 2]);
  }
  // The whole context's rows; row(h): the output row of column h, from out's first.
  template <typename Row>
  __device__ __forceinline__ void store(__nv_bfloat16* out, int cols, const Row& row) const {
    const int lane = threadIdx.x & 31, r = lane >> 2, c = lane & 3;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int h = 8 * t + 2 * c + x;
        if (h >= cols) continue;
        const float inv = 1.f / l[t][x];
        __nv_bfloat16* to = out + static_cast<int64_t>(row(h)) * D + 4 * r;
#pragma unroll
        for (int g = 0; g < GR; ++g) {
          const float4 v = four(t, g, x);
          *reinterpret_cast<uint2*>(to + 32 * g) =
              make_uint2(pack_bf16x2(v.x * inv, v.y * inv), pack_bf16x2(v.z * inv, v.w * inv));
        }
      }
  }
  // A part of one: O [heads][kStride], reference maxima and sums.
  template <int kStride>
  __device__ __forceinline__ void keep(float* part, float2* ml) const {
    const int lane = threadIdx.x & 31, r = lane >> 2, c = lane & 3;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int h = 8 * t + 2 * c + x;
#pragma unroll
        for (int g = 0; g < GR; ++g)
          *reinterpret_cast<float4*>(part + h * kStride + 32 * g + 4 * r) = four(t, g, x);
        if (r == 0) ml[h] = make_float2(m[t][x], l[t][x]);
      }
  }
};

// Parts joined, N at a time: O 2^(m - M) and sums, relative to the largest maximum yet.
struct Joined {
  float M = kNone, L = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  template <int N>
  __device__ __forceinline__ void add(const float2 (&ml)[N], const float4 (&v)[N]) {
    float top = M;
#pragma unroll
    for (int i = 0; i < N; ++i) top = fmaxf(top, ml[i].x);
    const float a = ex2_approx(M - top);
    M = top;
    L *= a;
    o.x *= a, o.y *= a, o.z *= a, o.w *= a;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float b = ex2_approx(ml[i].x - top);
      L = fmaf(ml[i].y, b, L);
      o.x = fmaf(v[i].x, b, o.x), o.y = fmaf(v[i].y, b, o.y);
      o.z = fmaf(v[i].z, b, o.z), o.w = fmaf(v[i].w, b, o.w);
    }
  }
  __device__ __forceinline__ void store(__nv_bfloat16* to) const {
    const float inv = 1.f / L;
    *reinterpret_cast<uint2*>(to) =
        make_uint2(pack_bf16x2(o.x * inv, o.y * inv), pack_bf16x2(o.z * inv, o.w * inv));
  }
};

}  // namespace dec
}  // namespace
}  // namespace gc

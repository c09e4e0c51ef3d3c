// The 4-bit cache: where a value is, and the maps between bf16 rows and stored ones.
//
// A row is one token's d columns of one kv head.  Groups of 32 columns share a scale:
//     s = bf16_rne(min(amax / 7, 2^15)), 0 if that is below 2^-24
//     c = clamp(rne(x * (1 / s)), -7, 7), every c = 0 when s = 0, c = 0 for NaN
// (amax over the group's finite values; quotients rounded once in binary32, the product
// only to the whole number), and c + 8 is stored in four bits.  The value is c s: 11
// significant bits, exact in binary32.  The rounding of s is a choice of the format: its 8
// bits cost a code at most 7 * 2^-8 of a step, and a scale takes two bytes.
//
// A (page, plane, kv head) has its rows' codes [ps][d/2] bytes, then their scales
// [ps][d/32] bf16.  The order of a row's codes is the one in which the decode kernel's
// threads hold them as operands of m16n8k16 products (decode_q4.cuh):
//     K: 32-bit word q * (d/32) + g holds columns 32 g + 8 q + j, q < 4; column j is in
//        nibble (0, 4, 2, 6, 1, 5, 3, 7)[j]
//     V: 16-bit word r * (d/32) + g holds columns 32 g + 4 r + j, r < 8, nibble j
#pragma once

#include "gc_internal.cuh"

namespace gc {

constexpr int kQ4Group = 32;  // columns that share a scale

// Bytes of one row, and of a head's rows of a page.
__host__ __device__ constexpr uint32_t q4_row_bytes(int d) { return d / 2 + d / 16; }
__host__ __device__ constexpr uint64_t q4_head_bytes(int d, int ps) {
  return static_cast<uint64_t>(ps) * q4_row_bytes(d);
}

// A cache with the geometry of a pool but pages of its own.
struct Q4Geom {
  uint8_t* cache;
  uint64_t head_bytes;
  int32_t pages, Hkv, ps, ps_shift;
};

__device__ __forceinline__ uint8_t* q4_head(const Q4Geom& g, int layer, int kv, int page, int h) {
  return g.cache +
         (((static_cast<uint64_t>(layer) * 2 + kv) * g.pages + page) * g.Hkv + h) * g.head_bytes;
}

namespace q4 {

__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("max.u16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
// a * b + c in binary32 pairs, rounded once
__device__ __forceinline__ void scale_add(uint32_t lo, uint32_t hi, uint64_t b, uint64_t c,
                                          uint32_t& x, uint32_t& y) {
  asm("{\n\t.reg .b64 t;\n\t"
      "mov.b64 t, {%2, %3};\n\t"
      "fma.rn.f32x2 t, t, %4, %5;\n\t"
      "mov.b64 {%0, %1}, t;\n\t}"
      : "=r"(x), "=r"(y)
      : "r"(lo), "r"(hi), "l"(b), "l"(c));
}

// |x| patterns of 8 bf16 values order like the magnitudes, non-finite ones on top.
__device__ __forceinline__ uint32_t abs_max8(const uint4& v) {
  const uint32_t m = 0x7fff7fffu;
  const uint32_t x = max_u16x2(max_u16x2(v.x & m, v.y & m), max_u16x2(v.z & m, v.w & m));
  return max(x & 0xffffu, x >> 16);
}
__device__ __forceinline__ uint32_t finite_abs_max8(const uint4& v) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t a = w[i / 2] >> 16 * (i & 1) & 0x7fffu;
    m = max(m, a < 0x7f80u ? a : 0u);
  }
  return m;
}

// Codes + 8 of 8 values as bytes: e has those of columns 0, 2, 4, 6, o of 1, 3, 5, 7.
// x / s + 1.5 * 2^23 + 8 is rounded to a whole number, ties to even, whose last bits are
// c + 8; |x / s| is at most 7.03 where s is neither clamped nor 0, so nothing is clamped.
__device__ __forceinline__ void codes8(const uint4& v, float inv, uint32_t& e, uint32_t& o) {
  const uint64_t inv2 = static_cast<uint64_t>(__float_as_uint(inv)) << 32 | __float_as_uint(inv);
  constexpr uint64_t magic = 0x4B4000084B400008ull;
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  uint32_t x[4], y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) scale_add(w[i] << 16, w[i] & 0xffff0000u, inv2, magic, x[i], y[i]);
  e = __byte_perm(__byte_perm(x[0], x[1], 0x0040), __byte_perm(x[2], x[3], 0x0040), 0x5410);
  o = __byte_perm(__byte_perm(y[0], y[1], 0x0040), __byte_perm(y[2], y[3], 0x0040), 0x5410);
}
// The same for any values.
__device__ __forceinline__ uint32_t code_any(uint32_t bits, float inv) {
  const float x = __uint_as_float(bits), p = x * inv;
  if (p != p) return 8;  // NaN, or infinity where s is 0
  if (fabsf(p) >= 8.f) return p > 0.f ? 15 : 1;
  const uint32_t u = __float_as_uint(fmaf(x, inv, 12582920.f)) & 0xffu;  // 0 to 16
  return min(max(u, 1u), 15u);
}
__device__ __forceinline__ void codes8_any(const uint4& v, float inv, uint32_t& e, uint32_t& o) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  e = o = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    e |= code_any(w[i] << 16, inv) << 8 * i;
    o |= code_any(w[i] & 0xffff0000u, inv) << 8 * i;
  }
}

// A row in the hands of four neighbouring lanes: lane q of them has the columns
// 32 g + 8 q ... + 7 of every group g as x[g].  All lanes of the warp call;
// those of `write` write the row's codes (16 bytes a lane at d = 128, 8 at 64) and scales.
template <int GR>
__device__ __forceinline__ void store_row(const uint4 (&x)[GR], bool is_k, uint8_t* codes,
                                          uint8_t* scales, bool write) {
  constexpr uint32_t all = 0xffffffffu;
  const int q = threadIdx.x & 3;
  uint32_t m[GR / 2];  // two groups' maxima each
#pragma unroll
  for (int i = 0; i < GR / 2; ++i) m[i] = abs_max8(x[2 * i]) | abs_max8(x[2 * i + 1]) << 16;
#pragma unroll
  for (int d = 1; d < 4; d <<= 1)
#pragma unroll
    for (int i = 0; i < GR / 2; ++i) m[i] = max_u16x2(m[i], __shfl_xor_sync(all, m[i], d));
  bool plain = true;
#pragma unroll
  for (int i = 0; i < GR / 2; ++i) plain &= (m[i] & 0xffffu) < 0x7f80u && m[i] < 0x7f800000u;
  if (__any_sync(all, !plain)) {
    uint32_t f[GR / 2];
#pragma unroll
    for (int i = 0; i < GR / 2; ++i) {
      f[i] = finite_abs_max8(x[2 * i]) | finite_abs_max8(x[2 * i + 1]) << 16;
#pragma unroll
      for (int d = 1; d < 4; d <<= 1) f[i] = max_u16x2(f[i], __shfl_xor_sync(all, f[i], d));
      m[i] = f[i];
    }
  }
  // lane q works out the scale of group q (at d = 64 the lanes 2 and 3 do it again)
  const int mine = q & (GR - 1);
  uint32_t amax = m[0];
#pragma unroll
  for (int i = 1; i < GR / 2; ++i)
    if (mine >> 1 == i) amax = m[i];
  amax = mine & 1 ? amax & 0xffff0000u : amax << 16;
  const float top = __uint_as_float(amax) / 7.0f;
  plain &= top <= 32768.0f;  // of this lane's group
  __nv_bfloat16 sb = __float2bfloat16_rn(fminf(top, 32768.0f));
  float s = __bfloat162float(sb);
  if (s < 5.9604644775390625e-8f) {
    s = 0.f;
    sb = __float2bfloat16_rn(0.f);
  }
  const float inv = s > 0.f ? 1.0f / s : 0.f;
  const bool fast = __all_sync(all, plain);
  uint32_t w[GR];
#pragma unroll
  for (int g = 0; g < GR; ++g) {
    const float i = __shfl_sync(all, inv, (threadIdx.x & 28) + g);
    uint32_t e, o;
    if (fast)
      codes8(x[g], i, e, o);
    else
      codes8_any(x[g], i, e, o);
    if (is_k) {
      // bytes (j0, j2, j1, j3) and (j4, j6, j5, j7)
      w[g] = __byte_perm(e, o, 0x5410) | __byte_perm(e, o, 0x7632) << 4;
    } else {
      w[g] = e | o << 4;  // columns 0-3 in the low half
    }
  }
  if (!write) return;
  if (!is_k) {
    if constexpr (GR == 4) {
      const uint32_t a = __byte_perm(w[0], w[1], 0x5410), b = __byte_perm(w[2], w[3], 0x5410);
      const uint32_t c = __byte_perm(w[0], w[1], 0x7632), d = __byte_perm(w[2], w[3], 0x7632);
      w[0] = a, w[1] = b, w[2] = c, w[3] = d;
    } else {
      const uint32_t a = __byte_perm(w[0], w[1], 0x5410);
      w[1] = __byte_perm(w[0], w[1], 0x7632);
      w[0] = a;
    }
  }
  if constexpr (GR == 4)
    reinterpret_cast<uint4*>(codes)[q] = make_uint4(w[0], w[1], w[2], w[3]);
  else
    reinterpret_cast<uint2*>(codes)[q] = make_uint2(w[0], w[1]);
  if (q < GR) reinterpret_cast<__nv_bfloat16*>(scales)[q] = sb;
}

// nibble pairs (bits 0-3 of both halves) of w as bf16 whole numbers -8..7
__device__ __forceinline__ uint32_t whole_pair(uint32_t w) {
  uint32_t d;
  const uint32_t biased = (w & 0x000f000fu) | 0x43004300u;  // 128 + nibble
  asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(biased), "r"(0x43084308u));
  return d;
}

// The inverse for the same four lanes: x[g] = bf16_rne(c s) of columns 32 g + 8 q ... + 7
// (a product of bf16 values, rounded once).
template <int GR>
__device__ __forceinline__ void load_row(const uint8_t* codes, const uint8_t* scales,
                                         uint32_t (&w)[GR], uint32_t (&s)[GR / 2]) {
  const int q = threadIdx.x & 3;
  if constexpr (GR == 4) {
    const uint4 v = ld_plain(reinterpret_cast<const uint4*>(codes) + q);
    const uint2 t = ld_plain(reinterpret_cast<const uint2*>(scales));
    w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
    s[0] = t.x, s[1] = t.y;
  } else {
    const uint2 v = ld_plain(reinterpret_cast<const uint2*>(codes) + q);
    w[0] = v.x, w[1] = v.y;
    s[0] = ld_plain(reinterpret_cast<const uint32_t*>(scales));
  }
}
template <int GR>
__device__ __forceinline__ void expand_row(const uint32_t (&w)[GR], const uint32_t (&s)[GR / 2],
                                           bool is_k, uint4 (&x)[GR]) {
#pragma unroll
  for (int g = 0; g < GR; ++g) {
    const uint32_t s2 = __byte_perm(s[g / 2], 0, g & 1 ? 0x3232 : 0x1010);
    if (is_k) {
      x[g].x = mul_bf16x2(whole_pair(w[g]), s2);
      x[g].y = mul_bf16x2(whole_pair(w[g] >> 8), s2);
      x[g].z = mul_bf16x2(whole_pair(w[g] >> 4), s2);
      x[g].w = mul_bf16x2(whole_pair(w[g] >> 12), s2);
    } else {
      // 16-bit word g of the units 2 q and 2 q + 1
      const uint32_t v = __byte_perm(w[g / 2], w[g / 2 + GR / 2], g & 1 ? 0x7632 : 0x5410);
      const uint32_t a = mul_bf16x2(whole_pair(v), s2), b = mul_bf16x2(whole_pair(v >> 4), s2);
      const uint32_t c = mul_bf16x2(whole_pair(v >> 8), s2);
      const uint32_t d = mul_bf16x2(whole_pair(v >> 12), s2);
      x[g].x = __byte_perm(a, b, 0x5410);
      x[g].y = __byte_perm(c, d, 0x5410);
      x[g].z = __byte_perm(a, b, 0x7632);
      x[g].w = __byte_perm(c, d, 0x7632);
    }
  }
}

}  // namespace q4
}  // namespace gc

// How decode in shares numbers its work with 32-bit ints, and the room that it needs
// (host arithmetic).
#pragma once
#include <cstddef>
#include <cstdint>
#include <initializer_list>

namespace gc {

// What a pair (request, kv head) costs beyond its keys, counted as keys in front of
// it: its look-ups and merge take a CTA about as long as 256 keys.  Shares of equal
// keys alone left the CTAs of the short contexts running when the others were done,
// SMs busy 75 % of the time on 64 multi-turn contexts over 8-bit pages (146 us; with
// 128, 256, 384 keys 131, 123, 124); one context of 9000 keys 19.1 us, now 16.2.
constexpr int kPairKeys = 256;

// Keys per unit as a shift, and the units in front of each pair's keys.
struct DecodeUnits {
  int shift, lead;
};

// For `pairs` pairs of at most `cap` keys, `margin` being what the kernel adds to
// the count.  Units of 16 keys where a 32-bit count can hold all of the block
// tables' capacity, of 128 keys otherwise, then with the allowance if it fits too.
inline DecodeUnits decode_units(int64_t pairs, int64_t cap, int64_t margin) {
  const int64_t per_pair = (INT32_MAX - margin) / pairs;  // units it may have
  for (const int shift : {4, 7}) {
    const int lead = kPairKeys >> shift;
    if (((cap - 1) >> shift) + 1 + lead <= per_pair) return {shift, lead};
  }
  return {7, 0};
}

// CTAs on an SM, or groups of a CTA, that decode with `heads` (8 or 16) q heads in registers:
// two where their accumulators leave room for both.
constexpr int decode_ctas(int head_dim, int heads) { return head_dim * heads <= 1024 ? 2 : 1; }

// Bytes of the partials of a call's shares: each CTA (or group) has two, of the heads' O and
// their maxima and sums, in binary32.  `per_kv_head` q heads, at most `most` CTAs.
inline size_t decode_share_bytes(int head_dim, int per_kv_head, int num_sms, int most) {
  const int heads = per_kv_head <= 8 ? 8 : 16, all = decode_ctas(head_dim, heads) * num_sms;
  return static_cast<size_t>(all < most ? all : most) * 2 * heads * (head_dim + 2) * sizeof(float);
}

}  // namespace gc

// What the own keys of requests behind shared prefixes cost where the SMs are divided
// between them and the prefixes (span.cuh); host and device arithmetic.
#pragma once
#include <cstdint>

#ifdef __CUDACC__
#define GC_HOST_DEVICE __host__ __device__
#else
#define GC_HOST_DEVICE
#endif

namespace gc {

// A request with a length outside [0, cap], the capacity of its block table, is skipped, so
// it costs nothing, like one without own keys.
GC_HOST_DEVICE inline bool own_keys_count(int32_t T, int32_t cap) { return T > 0 && T <= cap; }

// Of T keys in shares: T + 256, longer ones up to 1024 more (2 T between).  (T may be near
// 2^31, and thousands of them are summed up.)
GC_HOST_DEVICE inline int64_t own_keys_cost(int32_t T) {
  return static_cast<int64_t>(T) + (T < 256 ? 256 : T > 1024 ? 1024 : T);
}

// Of T keys where a pair goes to a warp, which takes at most `longest` of them.
GC_HOST_DEVICE inline int32_t own_keys_cost_by_warp(int32_t T, int32_t longest) {
  return (T < longest ? T : longest) + 48;
}

}  // namespace gc

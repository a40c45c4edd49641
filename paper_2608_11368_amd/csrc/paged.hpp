// Device helpers of the paged cache's kernels and of the gradient clipping.
#pragma once

#include "common.hpp"
#include "launch.hpp"

namespace pair {

// Division of 0 <= n < 2^31 by a fixed d >= 1 as a high product, an add and a
// shift (Granlund and Montgomery, PLDI '94): with s = ceil(log2 d) and
// m = floor(2^32 (2^s - d) / d) + 1, n / d = (mulhi(n, m) + n) >> s; the sum
// stays below 2^32 because n < 2^31.
struct FastDiv {
  uint32_t d, m, s;
};

inline FastDiv fast_div(uint32_t d) {
  uint32_t s = 0;
  while (s < 32 && ((uint64_t)1 << s) < d) ++s;
  const uint64_t m = (((((uint64_t)1 << s) - d) << 32) / d) + 1;
  return FastDiv{d, (uint32_t)m, s};
}

__device__ __forceinline__ uint32_t div_by(uint32_t n, const FastDiv& f) {
  return (__umulhi(n, f.m) + n) >> f.s;
}

// A wave-uniform value as a scalar.
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

__device__ __forceinline__ int64_t uniform64(int64_t v) {
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)v);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)((uint64_t)v >> 32));
  return (int64_t)(((uint64_t)hi << 32) | lo);
}

}  // namespace pair

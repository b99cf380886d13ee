// Ranking shared by the token filter and the cache eviction.
#pragma once
#include "common.cuh"

#ifdef __CUDACC__
namespace spv {

constexpr int kSelThreads = 1024;

// Larger value -> larger key.  +0 and -0 share a key; NaN gets key 0 (ranks last).
__device__ __forceinline__ uint32_t rank_key(float m) {
  if (m != m) return 0u;
  if (m == 0.0f) m = 0.0f;   // folds -0 into +0
  uint32_t u = __float_as_uint(m);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

}  // namespace spv
#endif

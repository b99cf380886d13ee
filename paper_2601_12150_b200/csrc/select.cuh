// Ranking parts shared by the token filter and the cache eviction.
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

// Block-wide exclusive scan of two counters; returns this thread's exclusive prefixes and the
// block totals.  Called by all kSelThreads threads.
__device__ __forceinline__ void block_scan2(int a, int b, int& ea, int& eb, int& ta, int& tb, int (*warp_tot)[2]) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int ia = a, ib = b;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    int na = __shfl_up_sync(0xffffffffu, ia, o), nb = __shfl_up_sync(0xffffffffu, ib, o);
    if (lane >= o) { ia += na; ib += nb; }
  }
  if (lane == 31) { warp_tot[warp][0] = ia; warp_tot[warp][1] = ib; }
  __syncthreads();
  if (warp == 0) {
    int wa = warp_tot[lane][0], wb = warp_tot[lane][1];
    int sa = wa, sb = wb;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      int na = __shfl_up_sync(0xffffffffu, sa, o), nb = __shfl_up_sync(0xffffffffu, sb, o);
      if (lane >= o) { sa += na; sb += nb; }
    }
    warp_tot[lane][0] = sa - wa;   // exclusive warp offsets
    warp_tot[lane][1] = sb - wb;
    if (lane == 31) { warp_tot[32][0] = sa; warp_tot[32][1] = sb; }
  }
  __syncthreads();
  ea = warp_tot[warp][0] + ia - a;
  eb = warp_tot[warp][1] + ib - b;
  ta = warp_tot[32][0];
  tb = warp_tot[32][1];
  __syncthreads();
}

}  // namespace spv
#endif

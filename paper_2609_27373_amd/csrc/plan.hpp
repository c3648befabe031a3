// plan.hpp — helpers of the work-groups that plan a launch: one group of 1024
// threads, so that prefix sums over all sequences of a call need no second launch.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace wise {

constexpr int kPlan = 1024;            // threads of a planning work-group
constexpr int kPlanWaves = kPlan / 64;

// Inclusive scan of x over the lanes of a wave on the VALU (DPP row shifts and
// broadcasts): a tenth of the latency of six LDS permutes.  op(a, b) with b = none
// changes nothing.
template <class Op>
__device__ __forceinline__ int wave_scan(int x, int none, Op op) {
  x = op(x, __builtin_amdgcn_update_dpp(none, x, 0x111, 0xF, 0xF, false));   // row_shr 1, 2, 4, 8
  x = op(x, __builtin_amdgcn_update_dpp(none, x, 0x112, 0xF, 0xF, false));
  x = op(x, __builtin_amdgcn_update_dpp(none, x, 0x114, 0xF, 0xF, false));
  x = op(x, __builtin_amdgcn_update_dpp(none, x, 0x118, 0xF, 0xF, false));
  x = op(x, __builtin_amdgcn_update_dpp(none, x, 0x142, 0xA, 0xF, false));   // row_bcast 15 into rows 1 and 3
  x = op(x, __builtin_amdgcn_update_dpp(none, x, 0x143, 0xC, 0xF, false));   // row_bcast 31 into rows 2 and 3
  return x;
}
__device__ __forceinline__ int wave_scan_add(int x) {
  return wave_scan(x, 0, [](int a, int b) { return a + b; });
}
__device__ __forceinline__ int wave_scan_max(int x) {
  return wave_scan(x, -0x7fffffff - 1, [](int a, int b) { return a > b ? a : b; });
}

// Sum over a wave of x < 2^44: two parts whose sums fit 32 bits.
__device__ __forceinline__ int64_t wave_total(int64_t x) {
  const int lo = wave_scan_add((int)(x & 0xfffff)), hi = wave_scan_add((int)(x >> 20));
  return (int64_t)__builtin_amdgcn_readlane(lo, 63) + ((int64_t)__builtin_amdgcn_readlane(hi, 63) << 20);
}

// Exclusive prefix sum of x over the group, and the total; waves: kPlanWaves
// words of LDS.
__device__ inline int64_t plan_scan(int64_t x, int64_t* total, int64_t* waves) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  // x < 2^44 in two parts whose sums over a wave fit 32 bits
  const int64_t s = (int64_t)wave_scan_add((int)(x & 0xfffff)) + ((int64_t)wave_scan_add((int)(x >> 20)) << 20);
  __syncthreads();
  if (lane == 63) waves[wave] = s;
  __syncthreads();
  int64_t before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kPlanWaves; ++w) {
    before += w < wave ? waves[w] : 0;
    all += waves[w];
  }
  *total = all;
  return before + s - x;
}

// Largest i with first[i] <= k, where first[0] = 0 and first ascends over its
// kN entries: the entry that holds place k.
template <int kN>
__device__ inline int plan_entry(const int32_t* first, int k) {
  int lo = 0, hi = kN;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (first[mid] <= k) lo = mid;
    else hi = mid;
  }
  return lo;
}

__device__ __forceinline__ bool in_range(int x, int n) { return (unsigned)x < (unsigned)n; }

}  // namespace wise

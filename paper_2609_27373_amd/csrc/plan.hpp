// plan.hpp — helpers of the work-groups that plan a launch: one group of 1024
// threads, so that prefix sums over all sequences of a call need no second launch.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace wise {

constexpr int kPlan = 1024;            // threads of a planning work-group
constexpr int kPlanWaves = kPlan / 64;

// Exclusive prefix sum of x over the group, and the total; waves: kPlanWaves
// words of LDS.
__device__ inline int64_t plan_scan(int64_t x, int64_t* total, int64_t* waves) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int64_t s = x;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t y = __shfl_up((long long)s, o, 64);
    if (lane >= o) s += y;
  }
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

// Largest i with first[i] <= k, where first[0] = 0 and first ascends over the
// group's kPlan entries: the entry that holds place k.
__device__ inline int plan_entry(const int32_t* first, int k) {
  int lo = 0, hi = kPlan;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (first[mid] <= k) lo = mid;
    else hi = mid;
  }
  return lo;
}

__device__ __forceinline__ bool in_range(int x, int n) { return (unsigned)x < (unsigned)n; }

}  // namespace wise

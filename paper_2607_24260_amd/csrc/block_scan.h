// Prefix sums over a workgroup, and the search in them.
#pragma once

#include "kap_internal.h"

namespace kap {

constexpr int kScanThreads = 1024, kScanWaves = kScanThreads / 64;

__device__ __forceinline__ long long wave_incl(long long x, int lane) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const long long y = __shfl_up(x, o, 64);
    if (lane >= o) x += y;
  }
  return x;
}

// Inclusive prefix sums of N values over a workgroup of kScanThreads, and their totals.
template <int N>
__device__ __forceinline__ void scan(const long long (&x)[N], long long (&incl)[N],
                                     long long (&total)[N], long long (*s)[kScanWaves]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int i = 0; i < N; ++i) incl[i] = wave_incl(x[i], lane);
  __syncthreads();                             // (the last scan's readers)
  if (lane == 63)
#pragma unroll
    for (int i = 0; i < N; ++i) s[i][wave] = incl[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const long long v = wave_incl(lane < kScanWaves ? s[i][lane] : 0, lane);
    total[i] = __shfl(v, 63, 64);
    incl[i] += wave > 0 ? __shfl(v, wave - 1, 64) : 0;
  }
}

// The last entry of n ascending ones that is at most k (the first is).
template <class T>
__device__ __forceinline__ int last_at_most(const T *first, int n, long long k) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (first[mid] <= k) lo = mid;
    else hi = mid;
  }
  return lo;
}

}  // namespace kap

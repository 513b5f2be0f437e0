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

// The same of whole numbers below 2^31, by row shifts.
__device__ __forceinline__ long long wave_incl_int(int x) {
  return ((long long)wave_scan_add(x >> 16) << 16) + wave_scan_add(x & 0xffff);
}
template <class T> __device__ __forceinline__ long long wave_incl_of(T x, int lane) {
  if constexpr (sizeof(T) == 4) return wave_incl_int(x);
  else return wave_incl(x, lane);
}

// Inclusive prefix sums of N values (not negative) over a workgroup of WAVES wavefronts, and
// their totals.
template <int N, int WAVES, class T>
__device__ __forceinline__ void scan(const T (&x)[N], long long (&incl)[N], long long (&total)[N],
                                     long long (*s)[WAVES]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int i = 0; i < N; ++i) incl[i] = wave_incl_of(x[i], lane);
  __syncthreads();                             // (the last scan's readers)
  if (lane == 63)
#pragma unroll
    for (int i = 0; i < N; ++i) s[i][wave] = incl[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const long long mine = lane < WAVES ? s[i][lane] : 0;
    long long before = mine;
#pragma unroll
    for (int o = 1; o < WAVES; o <<= 1) {
      const long long y = __shfl_up(before, o, 64);
      if (lane >= o) before += y;
    }
    total[i] = __shfl(before, WAVES - 1, 64);
    incl[i] += wave > 0 ? __shfl(before, wave - 1, 64) : 0;
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

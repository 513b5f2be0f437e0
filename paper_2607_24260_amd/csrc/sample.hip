// Drawing a token from logits filtered by temperature, top-k, top-p and min-p,
// with one given uniform number a row (the proposal's token, and the carry
// token after a window; Sec. 3.2 of the paper leaves the draw to the model).
//
// With w_i = exp((x_i - max) / T) and the tokens in descending order of their
// logits (ties: the lowest index first), every filter keeps a leading run:
//   top-k the first k; top-p the shortest run that holds p of the weight W of
//   the top-k run; min-p those with w_i >= min_p.
// The shortest of the three, N tokens, is drawn from: the first token at which
// the running weight exceeds u W(N).
//
// So every step asks at which token the running weight or count crosses a
// target. The weights are summed as integers, in units of 2^-s with
// s = 62 - ceil(log2 vocab): the sums do not depend on their order, and a
// running weight is off by less than vocab half units, where 32-bit floats
// would move the boundaries between tokens by as much as whole tokens.
#include "kap_internal.h"

#include <algorithm>

namespace kap {
namespace {

constexpr int kThreads = 1024;
constexpr int kBins = 256;

// Monotone map of a float to an unsigned key (-0 as +0, NaN as -inf).
__device__ __forceinline__ uint32_t order_key(float x) {
  if (x == 0.f) x = 0.f;
  if (x != x) x = -INFINITY;
  const uint32_t u = __float_as_uint(x);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t k) {
  return __uint_as_float((k & 0x80000000u) ? k ^ 0x80000000u : ~k);
}
constexpr uint32_t kNoKey = 0x007fffffu;   // -inf's: such a token is never drawn

// The weights of a row: exp2 in 64 bits of (x - max) * log2(e) / T.
struct Weights {
  float top;
  double slope;
  int bits;
  __device__ double of(uint32_t key) const {
    if (key == kNoKey) return 0.0;
    const float x = key_value(key);
    return x == top ? 1.0 : exp2(((double)x - (double)top) * slope);
  }
  __device__ unsigned long long units(double w) const {
    return (unsigned long long)rint(ldexp(w, bits));
  }
};

struct Shared {
  unsigned long long weight[kBins];
  unsigned long long red[kThreads / 64];
  int count[kBins];
  int pick[4];
};

template <typename T>
__device__ T block_max(T x, Shared &s) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) {
    const T y = __shfl_xor(x, o, 64);
    x = y > x ? y : x;
  }
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s.red[threadIdx.x >> 6] = x;
  __syncthreads();
  x = (T)s.red[0];
  for (int i = 1; i < kThreads / 64; ++i) x = (T)s.red[i] > x ? (T)s.red[i] : x;
  return x;
}

// A place in the descending order: the m-th (from 1) of the tokens with `key`,
// and the running weight and count up to and with it.
struct Place {
  uint32_t key;
  int m;
  unsigned long long weight;
  long long count;
};

template <int F32>
struct Row {
  const void *x;
  int n;
  __device__ uint32_t key(int i) const {
    if constexpr (F32) return order_key(static_cast<const float *>(x)[i]);
    return order_key(__uint_as_float((uint32_t)static_cast<const uint16_t *>(x)[i] << 16));
  }
};

// The first place whose running (weight, count) passes `cross`, by eight bits of
// the key at a time. It has to be passed at the end of the row.
template <int F32, class Cross>
__device__ Place descend(const Row<F32> &row, const Weights &wt, Shared &s, Cross cross) {
  Place p{0, 1, 0, 0};
  for (int shift = 24; shift >= 0; shift -= 8) {
    __syncthreads();
    for (int i = threadIdx.x; i < kBins; i += kThreads) {
      s.weight[i] = 0;
      s.count[i] = 0;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < row.n; i += kThreads) {
      const uint32_t k = row.key(i);
      if (shift < 24 && (k >> (shift + 8)) != (p.key >> (shift + 8))) continue;
      const int bin = (k >> shift) & (kBins - 1);
      atomicAdd(&s.count[bin], 1);
      atomicAdd(&s.weight[bin], wt.units(wt.of(k)));
    }
    __syncthreads();
    if (threadIdx.x == 0) {
      unsigned long long w = p.weight;
      long long c = p.count;
      int bin = kBins - 1, last = -1;
      for (; bin >= 0; --bin) {
        if (!s.count[bin]) continue;
        last = bin;
        if (cross(w + s.weight[bin], c + s.count[bin])) break;
        w += s.weight[bin];
        c += s.count[bin];
      }
      if (bin < 0) {           // not passed: the last token
        bin = last;
        w -= s.weight[bin];
        c -= s.count[bin];
      }
      s.pick[0] = bin;
      s.red[0] = w;
      s.red[1] = (unsigned long long)c;
      s.pick[1] = s.count[bin];
    }
    __syncthreads();
    p.key |= (uint32_t)s.pick[0] << shift;
    p.weight = s.red[0];
    p.count = (long long)s.red[1];
  }
  // s.pick[1] tokens have the key, of one weight each: the first of them that passes
  const unsigned long long unit = wt.units(wt.of(p.key));
  int lo = 1, hi = s.pick[1];
  while (lo < hi) {
    const int mid = lo + (hi - lo) / 2;
    if (cross(p.weight + mid * unit, p.count + mid)) hi = mid;
    else lo = mid + 1;
  }
  p.m = lo;
  p.weight += lo * unit;
  p.count += lo;
  return p;
}

// Index of the m-th token with `key`.
template <int F32>
__device__ int index_of(const Row<F32> &row, uint32_t key, int m, Shared &s) {
  int before = 0;
  for (int base = 0; base < row.n; base += kThreads) {
    const int i = base + threadIdx.x;
    const bool hit = i < row.n && row.key(i) == key;
    const unsigned long long b = __ballot(hit);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s.count[threadIdx.x >> 6] = __popcll(b);
    if (threadIdx.x == 0) s.pick[2] = -1;
    __syncthreads();
    int at = before, all = 0;
    for (int w = 0; w < kThreads / 64; ++w) {
      if (w < (int)(threadIdx.x >> 6)) at += s.count[w];
      all += s.count[w];
    }
    at += __popcll(b & ((1ull << (threadIdx.x & 63)) - 1)) + 1;
    if (hit && at == m) s.pick[2] = i;
    __syncthreads();
    if (s.pick[2] >= 0) return s.pick[2];
    before += all;
  }
  return -1;
}

template <int F32>
__global__ __launch_bounds__(kThreads) void sample_row_kernel(SampleArgs a) {
  __shared__ Shared s;
  const int r = blockIdx.x;
  const Row<F32> row{static_cast<const char *>(a.logits) + (size_t)r * a.stride * (F32 ? 4 : 2),
                     a.vocab};
  // the largest logit and the lowest index that has it
  unsigned long long best = 0;
  for (int i = threadIdx.x; i < row.n; i += kThreads) {
    const unsigned long long k = (unsigned long long)row.key(i) << 32 | (0xffffffffu - (uint32_t)i);
    best = k > best ? k : best;
  }
  best = block_max(best, s);
  const uint32_t top = (uint32_t)(best >> 32);
  int token = (int)(0xffffffffu - (uint32_t)best);
  float prob = 1.f;
  const float t = a.temperature ? a.temperature[r] : 1.f;
  if (top == kNoKey) {
    token = -1;
    prob = 0.f;
  } else if (t > 0.f) {
    const Weights wt{key_value(top), 1.4426950408889634074 / (double)t, a.bits};
    const int k = a.top_k && a.top_k[r] > 0 ? min(a.top_k[r], row.n) : row.n;
    const double p = a.top_p && a.top_p[r] < 1.f ? (double)a.top_p[r] : 1.0;
    const double q = a.min_p && a.min_p[r] > 0.f ? fmin((double)a.min_p[r], 1.0) : 0.0;
    double u = a.uniform[r];
    u = u > 0.0 ? fmin(u, 1.0 - 0x1p-24) : 0.0;
    Place cut = descend(row, wt, s, [&](unsigned long long, long long c) { return c >= k; });
    if (p < 1.0) {
      const double goal = p * (double)cut.weight;
      cut = descend(row, wt, s, [&](unsigned long long w, long long) { return (double)w >= goal; });
    }
    unsigned long long total = cut.weight;
    if (wt.of(cut.key) < q) {
      // min-p is the shortest run: the weights that reach it
      __syncthreads();
      if (threadIdx.x == 0) s.weight[0] = 0;
      __syncthreads();
      unsigned long long sum = 0;
      for (int i = threadIdx.x; i < row.n; i += kThreads) {
        const double w = wt.of(row.key(i));
        if (w >= q) sum += wt.units(w);
      }
      if (sum) atomicAdd(&s.weight[0], sum);
      __syncthreads();
      total = s.weight[0];
    }
    const double goal = u * (double)total;
    const Place at =
        descend(row, wt, s, [&](unsigned long long w, long long) { return (double)w > goal; });
    token = index_of(row, at.key, at.m, s);
    prob = (float)(ldexp(wt.of(at.key), a.bits) / (double)total);
  }
  if (threadIdx.x == 0) {
    a.token[r] = token;
    if (a.prob) a.prob[r] = prob;
  }
}

}  // namespace

hipError_t launch_sample(const SampleArgs &a, hipStream_t s) {
  if (a.f32)
    hipLaunchKernelGGL(sample_row_kernel<1>, dim3(a.rows), dim3(kThreads), 0, s, a);
  else
    hipLaunchKernelGGL(sample_row_kernel<0>, dim3(a.rows), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace kap

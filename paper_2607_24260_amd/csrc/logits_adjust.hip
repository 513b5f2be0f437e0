// Penalties for tokens that a row has had, biases, and a grammar's mask, on logits:
// one pass over the rows, in which a workgroup takes a slice of the vocabulary.
//
//   x <- x / r or x * r (x > 0 or not)   if the row's history holds the token
//   x <- x - f n - p                     n > 0 times among what the row has put out
//   x <- x + bias;  x <- -inf            where the mask's bit is 0
//
// What the history says of a slice is counted in LDS (integer atomics: the order
// does not matter), a word a token: how often the token was put out, and, in the
// top bit, whether the prompt has it. Biases go the same way, as the place in the list
// of the last one for the token. The slice's logits are fetched before the history is
// counted and meanwhile travel. Bound by the bytes: each logit is read and written once.
#include "kap_internal.h"

#include <algorithm>

namespace kap {
namespace {

constexpr int kThreads = 256;
constexpr uint32_t kPrompt = 0x80000000u;

template <bool F32> struct Elem { typedef float type; static constexpr int kPer = 4; };
template <> struct Elem<false> { typedef uint16_t type; static constexpr int kPer = 8; };

__device__ __forceinline__ float value(float x) { return x; }
__device__ __forceinline__ float value(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
template <class T> __device__ __forceinline__ T rounded(float x);
template <> __device__ __forceinline__ float rounded<float>(float x) { return x; }
// (to nearest: NaN stays NaN)
template <> __device__ __forceinline__ uint16_t rounded<uint16_t>(float x) {
  return __builtin_bit_cast(uint16_t, (__bf16)x);
}

// What a row asks for.
struct Row {
  float rep, freq, pres;
  bool told, biased;
  const uint32_t *mask;      // NULL: none
};

struct Slice {
  const uint32_t *counts;    // LDS, by token of the slice
  const int *biases;
  int v0;                    // first token
};

__device__ __forceinline__ float adjusted(const AdjustArgs &a, const Row &r, const Slice &s, float x,
                                          int v, bool allowed) {
  if (r.told) {
    const uint32_t c = s.counts[v - s.v0];
    if (c != 0) {
      x = x > 0.f ? x / r.rep : x * r.rep;
      const uint32_t n = c & ~kPrompt;
      if (n != 0) x = x - r.freq * (float)n - r.pres;
    }
  }
  if (r.biased) {
    const int e = s.biases[v - s.v0];
    if (e != 0) x += a.bias_value[e - 1];
  }
  return allowed ? x : -INFINITY;
}

// The mask's bits of tokens v .. v + 7 (those behind the last word: 0).
__device__ __forceinline__ uint32_t mask_bits(const uint32_t *mask, int words, int v) {
  const int w = v >> 5;
  const unsigned long long lo = mask[w], hi = w + 1 < words ? mask[w + 1] : 0u;
  return (uint32_t)((lo | hi << 32) >> (v & 31));
}

template <bool F32>
__global__ __launch_bounds__(kThreads) void adjust_logits_kernel(AdjustArgs a) {
  typedef typename Elem<F32>::type T;
  constexpr int kPer = Elem<F32>::kPer;
  extern __shared__ __align__(16) uint32_t lds[];
  const int row = blockIdx.y, v0 = blockIdx.x * a.slice, n = min(a.slice, a.vocab - v0);
  const int tid = threadIdx.x;
  uint32_t *counts = lds;
  int *biases = reinterpret_cast<int *>(lds + (a.history ? a.slice : 0));
  Row r;
  r.rep = a.repetition ? a.repetition[row] : 1.f;
  r.freq = a.frequency ? a.frequency[row] : 0.f;
  r.pres = a.presence ? a.presence[row] : 0.f;
  const int len = a.history ? max(a.history_len[row], 0) : 0;
  r.told = len > 0;
  int e0 = 0, e1 = 0;
  if (a.bias_offsets) {
    e0 = min(max(a.bias_offsets[row], 0), a.num_biases);
    e1 = min(max(a.bias_offsets[row + 1], e0), a.num_biases);
  }
  r.biased = e1 > e0;
  r.mask = nullptr;
  const int words = (a.vocab + 31) / 32;
  if (a.masks) {
    const int m = a.mask_row[row];
    if (m >= 0 && m < a.num_masks) r.mask = a.masks + (size_t)m * a.mask_stride;
  }
  if (r.told) {
    for (int i = tid; i < n; i += kThreads) counts[i] = 0;
  }
  if (r.biased) {
    for (int i = tid; i < n; i += kThreads) biases[i] = 0;
  }
  if (r.told || r.biased) __syncthreads();
  if (r.told) {
    // (a range outside the history counts where it is inside)
    const long long start = min(max((long long)a.history_start[row], -(1ll << 31)), a.history_size);
    const int prompt = a.prompt_len ? a.prompt_len[row] : 0;
    const long long lo = start < 0 ? -start : 0;
    const long long hi = min((long long)len, a.history_size - start);
    for (long long i = lo + tid; i < hi; i += kThreads) {
      const uint32_t at = (uint32_t)(a.history[start + i] - v0);
      if (at < (uint32_t)n) {
        if (i < prompt) atomicOr(&counts[at], kPrompt);
        else atomicAdd(&counts[at], 1u);
      }
    }
  }
  if (r.biased)
    for (int e = e0 + tid; e < e1; e += kThreads) {
      const uint32_t at = (uint32_t)(a.bias_token[e] - v0);
      if (at < (uint32_t)n) atomicMax(&biases[at], e + 1);
    }
  if (r.told || r.biased) __syncthreads();
  const Slice s{counts, biases, v0};
  const T *x = static_cast<const T *>(a.logits) + (size_t)row * a.stride + v0;
  T *y = static_cast<T *>(a.out) + (size_t)row * a.out_stride + v0;
  for (int i = tid; i < n; i += kThreads) {
    const int v = v0 + i;
    const bool allowed = !r.mask || (mask_bits(r.mask, words, v) & 1u);
    y[i] = rounded<T>(adjusted(a, r, s, value(x[i]), v, allowed));
  }
  (void)kPer;
}

}  // namespace

hipError_t launch_adjust_logits(AdjustArgs a, int cus, hipStream_t s) {
  a.slice = 8192;
  const int slices = (a.vocab + a.slice - 1) / a.slice;
  const size_t lds = (size_t)a.slice * 4 * ((a.history ? 1 : 0) + (a.bias_offsets ? 1 : 0));
  const dim3 grid(slices, a.rows), block(kThreads);
  if (a.f32) hipLaunchKernelGGL(adjust_logits_kernel<true>, grid, block, lds, s, a);
  else hipLaunchKernelGGL(adjust_logits_kernel<false>, grid, block, lds, s, a);
  return hipGetLastError();
}

}  // namespace kap

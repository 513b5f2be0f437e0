// Penalties for tokens that a row has had, biases, and a grammar's mask, on logits:
// one pass over the rows, in which a workgroup takes a slice of the vocabulary.
//
//   x <- x / r or x * r (x > 0 or not)   if the row's history holds the token
//   x <- x - f n - p                     n > 0 times among what the row has put out
//   x <- x + bias;  x <- -inf            where the mask's bit is 0
//
// What the history says of a slice is counted in LDS (integer atomics: the order
// does not matter), a word a token: how often the token was put out, and, in the
// top bit, whether the prompt has it. Tokens with a bias are marked there with a bit and
// left to the threads that walk the list; that the last of a token's entries counts
// takes a second look only where a slice's list names a token twice. The slice's logits
// are fetched first and travel while the history is counted. Bound by the bytes -- each
// logit is read and written once -- and by the history, which every slice of a row reads:
// 320 rows of 151937 bf16 logits with 4096 tokens 56 us, 3.5 TB/s (a large copy: 4.7; on the
// same tensors again and again, which the caches hold in part, 48.5 us, the others below too); 64
// of 151936 with 8192 tokens 18 us; one of 32000 in float32 4.5 us, the launch.
//   512 threads, two pieces of 16 bytes each, in 41 registers: four workgroups a compute
// unit (256 threads 52 us, 1024 65; four history loads in flight instead of two, for which
// only three workgroups fit, 54; 16 equal slices a row in one round of larger
// workgroups 59).
#include "kap_internal.h"

#include <algorithm>

namespace kap {
namespace {

constexpr int kThreads = 512;
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

constexpr int kBytes = 16;                     // of a thread's load
constexpr int kLoads = 2;                      // of a thread, at most
constexpr int kMost = kThreads * kLoads * kBytes / 2;   // tokens of a slice, at most

// What a row asks for.
struct Row {
  float rep, freq, pres;
  bool told;
  const uint32_t *mask;      // NULL: none
};

__device__ __forceinline__ float penalised(const Row &r, float x, uint32_t c) {
  if (c != 0) {
    x = x > 0.f ? x / r.rep : x * r.rep;
    const uint32_t n = c & ~kPrompt;
    if (n != 0) x = x - r.freq * (float)n - r.pres;
  }
  return x;
}

// Bits of tokens v .. v + 7 (those behind the last word: 0).
__device__ __forceinline__ uint32_t bits_at(const uint32_t *words, int n, int v) {
  const int w = v >> 5;
  const unsigned long long lo = words[w], hi = w + 1 < n ? words[w + 1] : 0u;
  return (uint32_t)((lo | hi << 32) >> (v & 31));
}

template <bool F32>
__global__ __launch_bounds__(kThreads, 8) void adjust_logits_kernel(AdjustArgs a) {
  typedef typename Elem<F32>::type T;
  constexpr int kPer = Elem<F32>::kPer;
  typedef T vec __attribute__((ext_vector_type(kPer)));
  constexpr int kSlice = kMost / (F32 ? 2 : 1);
  __shared__ __align__(16) uint32_t s_counts[kSlice + 4];
  __shared__ uint32_t s_biased[kSlice / 32], s_claimed[kSlice / 32];
  __shared__ int s_list[kThreads];
  __shared__ int s_twice;
  const int row = blockIdx.y, v0 = blockIdx.x * a.slice, n = min(a.slice, a.vocab - v0);
  const int tid = threadIdx.x;
  const T *x = static_cast<const T *>(a.logits) + (size_t)row * a.stride + v0;
  T *y = static_cast<T *>(a.out) + (size_t)row * a.out_stride + v0;
  // Whole 16-byte pieces where both rows have them at the same tokens, from the `skip`-th
  // token on; the rest one by one.
  const int skip_x = (int)(-(reinterpret_cast<uintptr_t>(x) / sizeof(T)) & (kPer - 1));
  const int skip_y = (int)(-(reinterpret_cast<uintptr_t>(y) / sizeof(T)) & (kPer - 1));
  const int skip = skip_x == skip_y ? min(skip_x, n) : n;
  const int pieces = (n - skip) / kPer;
  vec in[kLoads];
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const int p = tid + i * kThreads;
    if (p < pieces) in[i] = *reinterpret_cast<const vec *>(x + skip + p * kPer);
  }
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
  const bool biased = e1 > e0;
  r.mask = nullptr;
  const int words = (a.vocab + 31) / 32;
  if (a.masks) {
    const int m = a.mask_row[row];
    if (m >= 0 && m < a.num_masks) r.mask = a.masks + (size_t)m * a.mask_stride;
  }
  uint32_t allowed[kLoads];
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const int p = tid + i * kThreads;
    allowed[i] = r.mask && p < pieces ? bits_at(r.mask, words, v0 + skip + p * kPer) : ~0u;
  }
  // The history 16 bytes at a time, from the 16-byte boundary at or before its first token
  // on: tokens [before, end) from there, of which those below `prompt` are the prompt's.
  // (A range outside the history counts where it is inside.)
  typedef int i32x4 __attribute__((ext_vector_type(4)));
  constexpr int kAtOnce = 2;
  const int32_t *told = a.history;
  uint32_t before = 0, end = 0, prompt = 0;
  long long there = 0;                         // tokens from `told` on to the end of the array
  bool low = false;                            // and whether those before the first are in it
  if (r.told) {
    const long long start = min(max((long long)a.history_start[row], -(1ll << 31)), a.history_size);
    const long long lo = start < 0 ? -start : 0, hi = min((long long)len, a.history_size - start);
    const int32_t *first = a.history + start + lo;
    before = (uint32_t)(reinterpret_cast<uintptr_t>(first) / 4 & 3);
    told = first - before;
    end = hi > lo ? before + (uint32_t)(hi - lo) : 0;
    there = a.history_size - (start + lo) + before;
    low = start + lo >= before;
    const long long own = (long long)(a.prompt_len ? a.prompt_len[row] : 0) - lo + before;
    prompt = (uint32_t)min(max(own, 0ll), 0xffffffffll);
  }
  auto fetch = [&](i32x4 (&token)[kAtOnce], uint32_t j0) {
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const uint32_t j = j0 + 4 * k * kThreads;
      token[k] = i32x4{-1, -1, -1, -1};
      if (j >= end) continue;
      // (not across the ends of the array, though within a 16-byte line)
      if ((j >= before || low) && j + 4ll <= there) {
        token[k] = *reinterpret_cast<const i32x4 *>(told + j);
        if (j < before || j + 4 > end) {
#pragma unroll
          for (uint32_t c = 0; c < 4; ++c)
            if (j + c < before || j + c >= end) token[k][c] = -1;
        }
      } else {
#pragma unroll
        for (uint32_t c = 0; c < 4; ++c)
          if (j + c >= before && j + c < end) token[k][c] = told[j + c];
      }
    }
  };
  i32x4 token[kAtOnce];
  fetch(token, 4 * tid);
  const int e_own = e0 + tid, v_own = e_own < e1 ? a.bias_token[e_own] : -1;
  // (a piece's counts are 16-byte aligned in LDS)
  uint32_t *counts = s_counts + (-skip & 3);
  if (r.told) {
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    for (int i = 4 * tid; i < n + 4; i += 4 * kThreads)
      *reinterpret_cast<u32x4 *>(s_counts + i) = u32x4{0, 0, 0, 0};
  }
  if (biased) {
    for (int i = tid; i < (n + 31) / 32; i += kThreads) s_biased[i] = s_claimed[i] = 0;
    if (tid == 0) s_twice = 0;
  }
  if (r.told || biased) __syncthreads();
  for (uint32_t j0 = 4 * tid; j0 < end; j0 += 4 * kAtOnce * kThreads) {
    if (j0 != 4u * tid) fetch(token, j0);
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        // (n is at most 2^13 and v0 below 2^30: a negative token is far from both)
        const uint32_t at = (uint32_t)(token[k][c] - v0);
        if (at < (uint32_t)n) {
          if (j0 + 4 * k * kThreads + c < prompt) atomicOr(&counts[at], kPrompt);
          else atomicAdd(&counts[at], 1u);
        }
      }
  }
  if (biased)
    for (int e = e_own; e < e1; e += kThreads) {
      const int v = e == e_own ? v_own : a.bias_token[e];
      const uint32_t at = (uint32_t)(v - v0), bit = 1u << (at & 31);
      if (at < (uint32_t)n && (atomicOr(&s_biased[at >> 5], bit) & bit)) s_twice = 1;
    }
  if (r.told || biased) __syncthreads();

  // a token by itself (no bias: -0, which leaves every value as it is)
  auto write_one = [&](int at, float add) {
    const int v = v0 + at;
    float z = value(x[at]);
    if (r.told) z = penalised(r, z, counts[at]);
    z += add;
    if (r.mask && !(bits_at(r.mask, words, v) & 1u)) z = -INFINITY;
    y[at] = rounded<T>(z);
  };
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const int p = tid + i * kThreads;
    if (p >= pieces) continue;
    const int at = skip + p * kPer;
    constexpr uint32_t kAll = (1u << kPer) - 1;
    vec out = in[i];
    if (r.told) {
      typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
      u32x4 c[kPer / 4];
      uint32_t any = 0;
#pragma unroll
      for (int k = 0; k < kPer / 4; ++k) {
        c[k] = *reinterpret_cast<const u32x4 *>(counts + at + 4 * k);
        any |= c[k][0] | c[k][1] | c[k][2] | c[k][3];
      }
      if (any != 0) {
#pragma unroll
        for (int k = 0; k < kPer; ++k)
          out[k] = rounded<T>(penalised(r, value((T)out[k]), c[k >> 2][k & 3]));
      }
    }
    if (r.mask) {
#pragma unroll
      for (int k = 0; k < kPer; ++k)
        if (!(allowed[i] >> k & 1u)) out[k] = rounded<T>(-INFINITY);
    }
    const uint32_t left = biased ? bits_at(s_biased, (n + 31) / 32, at) & kAll : 0;
    if (left == 0) {
      *reinterpret_cast<vec *>(y + at) = out;
    } else {
#pragma unroll
      for (int k = 0; k < kPer; ++k)
        if (!(left >> k & 1u)) y[at + k] = out[k];
    }
  }
  for (int i = tid; i < n - pieces * kPer; i += kThreads) {
    const int at = i < skip ? i : i + pieces * kPer;
    if (!biased || !(s_biased[at >> 5] >> (at & 31) & 1u)) write_one(at, -0.f);
  }
  if (!biased) return;
  if (!s_twice) {
    for (int e = e_own; e < e1; e += kThreads) {
      const uint32_t at = (uint32_t)((e == e_own ? v_own : a.bias_token[e]) - v0);
      if (at < (uint32_t)n) write_one((int)at, a.bias_value[e]);
    }
    return;
  }
  // from the end of the list, as many entries at a time as there are threads: an entry
  // counts if none behind it has claimed its token, here or before
  for (int last = e1; last > e0; last -= kThreads) {
    const int e = last - 1 - tid;              // (thread 0 has the last)
    const int v = e >= e0 ? a.bias_token[e] : -1;
    const uint32_t at = (uint32_t)(v - v0);
    const bool in_slice = at < (uint32_t)n;
    s_list[tid] = in_slice ? (int)at : -1;
    __syncthreads();
    bool counts_here = in_slice && !(s_claimed[at >> 5] >> (at & 31) & 1u);
    for (int k = 0; k < tid && counts_here; ++k) counts_here = s_list[k] != (int)at;
    __syncthreads();
    if (counts_here) {
      atomicOr(&s_claimed[at >> 5], 1u << (at & 31));
      write_one((int)at, a.bias_value[e]);
    }
  }
}

}  // namespace

hipError_t launch_adjust_logits(AdjustArgs a, int cus, hipStream_t s) {
  // a workgroup's logits: 16 KB, or less where that would leave compute units idle
  const int most = a.f32 ? kMost / 2 : kMost;
  a.slice = most;
  while (a.slice > most / 8 && (long long)a.rows * ((a.vocab + a.slice - 1) / a.slice) < 2ll * cus)
    a.slice /= 2;
  const dim3 grid((a.vocab + a.slice - 1) / a.slice, a.rows), block(kThreads);
  if (a.f32) hipLaunchKernelGGL(adjust_logits_kernel<true>, grid, block, 0, s, a);
  else hipLaunchKernelGGL(adjust_logits_kernel<false>, grid, block, 0, s, a);
  return hipGetLastError();
}

}  // namespace kap

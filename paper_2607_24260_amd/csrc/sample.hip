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
// target. Nothing is sorted but the few tokens around the answers, in three
// launches over (row, chunk of the vocabulary):
//   1  the largest and smallest logit of every chunk;
//   2  a histogram of weights and counts over 2048 bins of equal ratio, from the
//      largest weight down to the smallest, or to 2^-32 (one bin for what is less);
//   3  from the running sums of the bins, those that an answer can lie in; their
//      tokens are collected, and the last workgroup of the row sorts them and
//      finds the answers among them.
// Rows for which that is not few tokens are descended eight bits of the logit at a
// time over the whole row instead, by the same last workgroup: thousands of equal
// logits around an answer, and bf16 logits far from zero are that (some -1e4 besides,
// high temperatures and 256K tokens make it likelier: bins are as wide as the smallest
// logit asks for), or a draw from weights below 2^-32. 64 rows of 151936 equal logits
// take 1.0 to 1.5 ms (equal logits are added up by the wavefront, 2.3 to 3.4 ms
// otherwise), of bf16 logits with mean 30 and deviation 2 1.3 to 1.9.
//
// The weights are summed as integers, in units of 2^-s with s = min(51, 62 - ceil(log2
// vocab)): the sums do not depend on their order, and a running weight is off by less
// than half a unit for each of its tokens (a unit for those below the last bin) and
// 2^-44 of itself for the exponentials, where 32-bit floats would move the boundaries
// between tokens by as much as whole tokens.
//
// Each launch reads the logits once (the later ones mostly from the caches). It is not
// bytes that bound it: the first launch goes at 2.7 TB/s for 64 x 151936 bf16 logits
// (7.1 us), the second computes weights (19.6 us), and the third is a chain of short
// steps of a row (20 us: sums of the bins 3, search 3, collecting 5, then the last
// workgroup's sort, sums and answers), of which few rows have no others to hide it
// behind. 46 us in all; 320 x 151937 112 us (0.9 TB/s), 16 x 128000 float32 30 us,
// 1 x 32000 float32 17 to 23 us (by the draw).
#include "kap_internal.h"

#include <algorithm>
#include <type_traits>

namespace kap {
namespace {

constexpr int kSumThreads = 512;               // of the first two launches
// Of the third: half as many as a CU takes at its registers, so that one row's chain
// falls into another's (1024: 1 row 18.6 for 17.1 us, 64 rows 45.6 for 44.8, 320 rows
// 118 for 112; 256: 16.4, 51, 136; rows of equal logits 0.8, 1.1 and 1.8 ms).
constexpr int kThreads = 512;
constexpr int kSampleWaves = kThreads / 64;
// A factor of two in weight has 32 steps, and a step a power of two of bins, two at
// least (2048 bins then reach down to 2^-32) and kFinest at most: as many as the
// row's smallest logit allows. 150K logits a few factors apart would else put
// thousands into a bin.
constexpr int kPerOctave = 32;
constexpr int kFinest = 64;
constexpr int kBins = 2048;
constexpr int kMost = 2048;                    // tokens sorted for a row

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
constexpr uint32_t kNoKey = 0x007fffffu;       // -inf's: such a token is never drawn

typedef unsigned long long u64;

// A token in the descending order: key above inverted index.
__device__ __forceinline__ u64 token_of(uint32_t key, int i) {
  return (u64)key << 32 | (0xffffffffu - (uint32_t)i);
}
__device__ __forceinline__ int index_of(u64 token) { return (int)(0xffffffffu - (uint32_t)token); }

// ---------------------------------------------------------------------------
// a row's tokens
// ---------------------------------------------------------------------------

template <int F32>
struct Row {
  static constexpr int kVec = F32 ? 4 : 8;     // logits of a 16-byte load
  const char *x;
  int n, head, vecs;                           // tokens before the first aligned load; loads
  __device__ Row(const SampleArgs &a, int r) {
    x = static_cast<const char *>(a.logits) + (size_t)r * a.stride * (F32 ? 4 : 2);
    n = a.vocab;
    head = min(n, (int)((-reinterpret_cast<uintptr_t>(x) & 15) / (F32 ? 4 : 2)));
    vecs = (n - head) / kVec;
  }
  __device__ float one(int i) const {
    if constexpr (F32) return reinterpret_cast<const float *>(x)[i];
    return __uint_as_float((uint32_t) reinterpret_cast<const uint16_t *>(x)[i] << 16);
  }
  // f(logits, index of the first) for the tokens of a chunk, kVec or one at a time,
  // a thread's tokens in ascending order. The next load is on its way meanwhile.
  template <int THREADS, class F>
  __device__ __forceinline__ void each(int chunk, int chunks, F f) const {
    auto single = [&](int i) {
      const float y[1] = {one(i)};
      f(y, i);
    };
    if (chunk == 0 && (int)threadIdx.x < head) single(threadIdx.x);
    const kv_u32x4 *v = reinterpret_cast<const kv_u32x4 *>(x + (size_t)head * (F32 ? 4 : 2));
    const int per = (vecs + chunks - 1) / chunks;
    const int v0 = chunk * per, v1 = min(vecs, v0 + per);
    if (v0 < v1) {
      int j = v0 + threadIdx.x;
      kv_u32x4 w = v[min(j, v1 - 1)];
      for (; j < v1; j += THREADS) {
        const kv_u32x4 next = v[min(j + THREADS, v1 - 1)];   // (past the end: the last again)
        float y[kVec];
#pragma unroll
        for (int e = 0; e < kVec; ++e)
          y[e] = F32 ? __uint_as_float(w[e & 3])
                     : ((e & 1) ? bf16_hi(w[(e >> 1) & 3]) : bf16_lo(w[(e >> 1) & 3]));
        f(y, head + j * kVec);
        w = next;
      }
    }
    if (chunk == chunks - 1) {
      const int i = head + vecs * kVec + (int)threadIdx.x;
      if (i < n) single(i);
    }
  }
};
// ---------------------------------------------------------------------------
// weights
// ---------------------------------------------------------------------------

// exp2 in 64 bits of (x - max) * log2(e) / T.
struct Weights {
  float top;
  double slope;
  int bits;
  __device__ double of(uint32_t key) const {
    if (key == kNoKey) return 0.0;
    const float x = key_value(key);
    return x == top ? 1.0 : exp2(((double)x - (double)top) * slope);
  }
  __device__ u64 units(double w) const { return (u64)rint(ldexp(w, bits)); }
};

// The same to 2^-44 of a weight, and its bin, for the sums over whole rows: with
// y = log2 w in bins and n = rint(y), 2^n from a table with a bin's weight each,
// times 2^(y - n) by its series to the fourth power (a bin is at most 1/64 of a
// factor of two: (ln 2 / 128)^5 / 5! = 2^-44.5). Eleven 64-bit operations and about
// thirty others a logit are what the second launch takes its time for: 64 rows of
// 151936 logits 19.5 us, of which 12.7 us are this loop, and 18.8 us without its LDS
// additions (splitting off whole factors of two and 32nds instead, with the fifth
// power: fifteen 64-bit operations).
struct FastWeights {
  double top, least, slope;                    // y = z * slope, z = x - top, least at least
  double c1, c2, c3, c4;                       // of 2^(y - n)
  int beyond;                                  // bits to shift a weight below the last bin by
  __device__ static constexpr double magic() { return 6755399441055744.0; }   // 1.5 * 2^52
  // z: 0 for the largest logit and not above it for any other, at any slope. (Of
  // x * slope - top * slope the rounding of a product is left, hundreds of bins at a
  // temperature of 1e-15.) y is -2 kBins + 1 at least: no unit is left of such a weight
  // (NaN's and -inf's too).
  __device__ double below(float x) const { return fmax((double)x - top, least); }
  __device__ double nearest(double z) const { return fma(z, slope, magic()); }   // low half: rint(y)
  __device__ static int bin(double t) { return -(int)(uint32_t)__double_as_longlong(t); }
  // units of a weight in bin b, of which 2^n has `unit`; t: nearest(z)
  __device__ u64 units(double z, double t, int b, double unit) const {
    const double f = fma(z, slope, magic() - t);
    const double p = fma(f, fma(f, fma(f, fma(f, c4, c3), c2), c1), 1.0);
    const u64 v = (u64)__double_as_longlong(fma(unit, p, 4503599627370496.0)) & 0xfffffffffffffull;
    return v >> (b >= kBins ? beyond : 0);
  }
  __device__ int bin_of(float x) const { return bin(nearest(below(x))); }
  // the units of 2^n in bin b (those below the last bin are a bin 2048 above, shifted)
  __device__ double unit_of(int b, int bits) const {
    return ldexp(exp2((b & (kBins - 1)) * (c1 * -1.4426950408889634074)), bits);
  }
};

__device__ __forceinline__ FastWeights fast_weights(float top, float low, float t) {
  // (not 0 at an infinite temperature, so that -inf stays apart)
  const double steps = fmax(kPerOctave * 1.4426950408889634074 / (double)t, 1e-300);
  const double span = ((double)top - (double)low) * steps + 1.0;
  double fine = 2.0;
  while (fine < kFinest && span * (2 * fine) < kBins) fine *= 2;
  const double slope = steps * fine, c = 0.69314718055994530942 / (kPerOctave * fine);
  // (with finer bins none of the row's tokens is below the last one)
  return FastWeights{top, (1.0 - 2 * kBins) / slope, slope, c, c * c / 2, c * c * c / 6,
                     c * c * c * c / 24, fine == 2.0 ? kBins / (2 * kPerOctave) : 63};
}

// What a row asks for. (An array that is not there is read as another one and the
// value left out: the loads go out together.)
struct Wants {
  float t;
  int k;             // vocab: no top-k
  double p, q, u;    // p 1: no top-p; q 0: no min-p
};
__device__ __forceinline__ Wants wants_of(const SampleArgs &a, int r) {
  const float u = a.uniform[r];
  const float t = (a.temperature ? a.temperature : a.uniform)[r];
  const int k = (a.top_k ? a.top_k : reinterpret_cast<const int32_t *>(a.uniform))[r];
  const float p = (a.top_p ? a.top_p : a.uniform)[r], q = (a.min_p ? a.min_p : a.uniform)[r];
  Wants w;
  w.t = a.temperature ? t : 1.f;
  w.k = a.top_k && k > 0 ? min(k, a.vocab) : a.vocab;
  w.p = a.top_p && p < 1.f ? (double)p : 1.0;
  w.q = a.min_p && q > 0.f ? fmin((double)q, 1.0) : 0.0;
  w.u = u > 0.f ? fmin((double)u, 1.0 - 0x1p-24) : 0.0;
  return w;
}

// The largest token and the smallest logit of a row from its chunks' (every
// wavefront by itself).
struct Ends {
  u64 best;
  float low;
};
__device__ __forceinline__ Ends row_ends(const SampleArgs &a, int r) {
  Ends e{0, INFINITY};
  for (int c = threadIdx.x & 63; c < a.chunks; c += 64) {
    e.best = max(e.best, a.tops[(size_t)r * a.chunks + c]);
    e.low = fminf(e.low, a.lows[(size_t)r * a.chunks + c]);
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) {
    e.best = max(e.best, __shfl_xor(e.best, o, 64));
    e.low = fminf(e.low, __shfl_xor(e.low, o, 64));
  }
  return e;
}

// Whether a row is drawn from, and whether by bins: its largest logit and
// temperature give finite coefficients.
__device__ __forceinline__ bool drawn(const Wants &w) { return w.t > 0.f; }
__device__ __forceinline__ bool by_bins(const Wants &w, uint32_t top) {
  return w.t > 1e-30f && key_value(top) < INFINITY;
}

// ---------------------------------------------------------------------------
// 1: the largest logit of every chunk; the row's sums are cleared
// ---------------------------------------------------------------------------

template <int F32>
__global__ __launch_bounds__(kSumThreads) void sample_top_kernel(SampleArgs a) {
  __shared__ u64 s_best[kSumThreads / 64];
  __shared__ float s_low[kSumThreads / 64];
  const int chunk = blockIdx.x, r = blockIdx.y;
  const Row<F32> row(a, r);
  float best = -INFINITY, low = INFINITY;      // low: of those above -inf
  int at = -1;
  row.template each<kSumThreads>(chunk, a.chunks, [&](const auto &x, int i) {
#pragma unroll
    for (int e = 0; e < (int)(sizeof(x) / sizeof(float)); ++e) {
      if (x[e] > best) {
        best = x[e];
        at = i + e;
      }
      low = fminf(low, x[e] == -INFINITY ? INFINITY : x[e]);
    }
  });
  u64 token = at < 0 ? 0 : token_of(order_key(best), at);
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) {
    token = max(token, __shfl_xor(token, o, 64));
    low = fminf(low, __shfl_xor(low, o, 64));
  }
  if ((threadIdx.x & 63) == 0) {
    s_best[threadIdx.x >> 6] = token;
    s_low[threadIdx.x >> 6] = low;
  }
  for (int i = chunk * kSumThreads + threadIdx.x; i <= kBins; i += a.chunks * kSumThreads) {
    a.weight[(size_t)r * (kBins + 1) + i] = 0;
    a.count[(size_t)r * (kBins + 1) + i] = 0;
  }
  if (chunk == 0 && threadIdx.x == 0) a.state[r] = 0;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < kSumThreads / 64; ++w) {
      token = max(token, s_best[w]);
      low = fminf(low, s_low[w]);
    }
    a.tops[(size_t)r * a.chunks + chunk] = token;
    a.lows[(size_t)r * a.chunks + chunk] = low;
  }
}

// ---------------------------------------------------------------------------
// 2: weights and counts by bin
// ---------------------------------------------------------------------------

template <int F32>
__global__ __launch_bounds__(kSumThreads) void sample_bins_kernel(SampleArgs a) {
  __shared__ u64 s_weight[kBins + 1];
  __shared__ int s_count[kBins + 1];
  __shared__ double s_unit[kBins];
  const int chunk = blockIdx.x, r = blockIdx.y;
  const Wants want = wants_of(a, r);
  const Ends ends = row_ends(a, r);
  const uint32_t top = (uint32_t)(ends.best >> 32);
  if (top == 0 || !by_bins(want, top)) return;
  const FastWeights w = fast_weights(key_value(top), ends.low, want.t);
  for (int i = threadIdx.x; i < kBins; i += kSumThreads) {
    s_weight[i] = 0;
    s_count[i] = 0;
    s_unit[i] = w.unit_of(i, a.bits);
  }
  if (threadIdx.x == 0) {
    s_weight[kBins] = 0;
    s_count[kBins] = 0;
  }
  __syncthreads();
  const bool counts = want.k < a.vocab;
  u64 rest = 0;
  int rest_n = 0;
  const Row<F32> row(a, r);
  row.template each<kSumThreads>(chunk, a.chunks, [&](const auto &x, int) {
    // (four at a time: eight take the registers of two wavefronts)
    constexpr int ALL = sizeof(x) / sizeof(float), N = ALL < 4 ? ALL : 4;
#pragma unroll
    for (int e0 = 0; e0 < ALL; e0 += N) {
      if (e0) __builtin_amdgcn_sched_barrier(0);
      int b[N];
      u64 v[N];
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const double z = w.below(x[e0 + e]), t = w.nearest(z);
        b[e] = FastWeights::bin(t);
        v[e] = w.units(z, t, b[e], s_unit[b[e] & (kBins - 1)]);
      }
#pragma unroll
      for (int e = 0; e < N; ++e) {
        // (the many below stay in registers; above the top there is nothing, unless the
        // row is written to meanwhile)
        const bool in = (uint32_t)b[e] < (uint32_t)kBins;
        rest += in ? 0 : v[e];
        rest_n += !in;
        if (in) atomicAdd(&s_weight[b[e]], v[e]);
      }
      if (counts) {
#pragma unroll
        for (int e = 0; e < N; ++e)
          if ((uint32_t)b[e] < (uint32_t)kBins) atomicAdd(&s_count[b[e]], 1);
      }
    }
  });
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) {
    rest += __shfl_xor(rest, o, 64);
    rest_n += __shfl_xor(rest_n, o, 64);
  }
  if ((threadIdx.x & 63) == 0) {
    atomicAdd(&s_weight[kBins], rest);
    atomicAdd(&s_count[kBins], rest_n);
  }
  __syncthreads();
  u64 *gw = a.weight + (size_t)r * (kBins + 1);
  int *gc = a.count + (size_t)r * (kBins + 1);
  for (int i = threadIdx.x; i <= kBins; i += kSumThreads) {
    if (s_weight[i]) atomicAdd(gw + i, s_weight[i]);
    if (counts && s_count[i]) atomicAdd(gc + i, s_count[i]);
  }
}

// ---------------------------------------------------------------------------
// 3: the answers
// ---------------------------------------------------------------------------

struct Shared {
  u64 weight[kBins + 1];                       // running, by bin
  int count[kBins + 1];
  u64 token[2][kMost];                         // collected, and sorted: descending;
                                               // then, in the place of the former,
                                               // running units of the sorted tokens
  uint16_t start[kBins + 1], stop[kBins + 1];  // a bin's sorted tokens
  uint32_t wanted[kBins / 32];
  u64 red[kSampleWaves];
  int red_n[kSampleWaves];
  int pick[4];
};

// First index in [lo, hi) at which f (false, then true) holds, else hi; by a
// whole wavefront, 64 strides at a time.
template <class F>
__device__ __forceinline__ int first_of(int lo, int hi, F f) {
  const int lane = threadIdx.x & 63;
  while (hi - lo > 64) {
    const int step = (hi - lo + 63) / 64;
    const int i = min(lo + (lane + 1) * step, hi) - 1;   // the last of a stretch
    const u64 hit = __ballot(f(i));
    if (!hit) return hi;
    const int l = __builtin_ctzll(hit);
    const int a = lo + l * step;
    hi = min(a + step, hi);
    lo = a;
  }
  const u64 hit = __ballot(lo + lane < hi && f(lo + lane));
  return hit ? lo + __builtin_ctzll(hit) : hi;
}

template <typename T>
__device__ __forceinline__ T wave_run(T v) {   // inclusive running sum over the lanes
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const T y = __shfl_up(v, o, 64);
    if (lane >= o) v += y;
  }
  return v;
}

// Running sums of the bins' weights and (HAS_K) counts: a thread has a few neighbouring bins.
constexpr int kOwnBins = kBins / kThreads;
template <bool HAS_K>
__device__ __forceinline__ void run_bins(const u64 *gw, const int *gc, Shared &s) {
  const int i = kOwnBins * threadIdx.x, wave = threadIdx.x >> 6;
  u64 w[kOwnBins];
  int c[kOwnBins];
#pragma unroll
  for (int e = 0; e < kOwnBins; ++e) {
    w[e] = gw[i + e];
    c[e] = HAS_K ? gc[i + e] : 0;
  }
  const u64 w_rest = gw[kBins];
  const int c_rest = HAS_K ? gc[kBins] : 0;
#pragma unroll
  for (int e = 1; e < kOwnBins; ++e) {
    w[e] += w[e - 1];
    c[e] += c[e - 1];
  }
  const u64 w_run = wave_run(w[kOwnBins - 1]);
  const int c_run = HAS_K ? wave_run(c[kOwnBins - 1]) : 0;
  if ((threadIdx.x & 63) == 63) {
    s.red[wave] = w_run;
    s.red_n[wave] = c_run;
  }
  __syncthreads();
  u64 w_at = w_run - w[kOwnBins - 1], w_all = 0;
  int c_at = c_run - c[kOwnBins - 1], c_all = 0;
  for (int v = 0; v < kSampleWaves; ++v) {
    if (v < wave) {
      w_at += s.red[v];
      c_at += s.red_n[v];
    }
    w_all += s.red[v];
    c_all += s.red_n[v];
  }
#pragma unroll
  for (int e = 0; e < kOwnBins; ++e) {
    s.weight[i + e] = w_at + w[e];
    if (HAS_K) s.count[i + e] = c_at + c[e];
  }
  if (threadIdx.x == 0) {
    s.weight[kBins] = w_all + w_rest;
    s.count[kBins] = c_all + c_rest;
  }
  __syncthreads();
}

// Inclusive running sums over n values of LDS, in place.
__device__ __forceinline__ void run_sums(u64 *x, int n, Shared &s) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  u64 before = 0;
  for (int base = 0; base < n; base += kThreads) {
    const int i = base + threadIdx.x;
    const u64 v = wave_run(i < n ? x[i] : 0);
    __syncthreads();
    if (lane == 63) s.red[wave] = v;
    __syncthreads();
    u64 add = before;
    for (int w = 0; w < kSampleWaves; ++w) {
      if (w < wave) add += s.red[w];
      before += s.red[w];
    }
    if (i < n) x[i] = v + add;
  }
  __syncthreads();
}

// ---- the whole row, eight bits of the key at a time ---------------------------

constexpr int kDigits = 256;

// A place in the descending order: the m-th (from 1) of the tokens with `key`,
// and the running weight up to and with it.
struct Place {
  uint32_t key;
  int m;
  u64 weight;
  long long count;
};

template <int F32, class Cross>
__device__ Place descend(const Row<F32> &row, const Weights &wt, Shared &s, Cross cross) {
  Place p{0, 1, 0, 0};
  for (int shift = 24; shift >= 0; shift -= 8) {
    __syncthreads();
    for (int i = threadIdx.x; i < kDigits; i += kThreads) {
      s.weight[i] = 0;
      s.count[i] = 0;
    }
    __syncthreads();
    row.template each<kThreads>(0, 1, [&](const auto &x, int) {
#pragma unroll 1
      for (int e = 0; e < (int)(sizeof(x) / sizeof(float)); ++e) {
        const uint32_t k = order_key(x[e]);
        if (shift < 24 && (k >> (shift + 8)) != (p.key >> (shift + 8))) continue;
        const int bin = (k >> shift) & (kDigits - 1);
        // (equal logits, which are what brings rows here, in one addition)
        const u64 here = __ballot(true);
        if (__ballot(k == (uint32_t)__builtin_amdgcn_readfirstlane((int)k)) == here) {
          if ((threadIdx.x & 63) == __builtin_ctzll(here)) {
            const int n = __popcll(here);
            atomicAdd(&s.count[bin], n);
            atomicAdd(&s.weight[bin], (u64)n * wt.units(wt.of(k)));
          }
          continue;
        }
        atomicAdd(&s.count[bin], 1);
        atomicAdd(&s.weight[bin], wt.units(wt.of(k)));
      }
    });
    __syncthreads();
    if (threadIdx.x == 0) {
      u64 w = p.weight;
      long long c = p.count;
      int bin = kDigits - 1, last = -1;
      for (; bin >= 0; --bin) {
        if (!s.count[bin]) continue;
        last = bin;
        if (cross(w + s.weight[bin], c + s.count[bin])) break;
        w += s.weight[bin];
        c += s.count[bin];
      }
      if (bin < 0) {                           // not passed: the last token
        bin = last;
        w -= s.weight[bin];
        c -= s.count[bin];
      }
      s.pick[0] = bin;
      s.red[0] = w;
      s.red[1] = (u64)c;
      s.pick[1] = s.count[bin];
    }
    __syncthreads();
    p.key |= (uint32_t)s.pick[0] << shift;
    p.weight = s.red[0];
    p.count = (long long)s.red[1];
  }
  // s.pick[1] tokens have the key, of one weight each: the first of them that passes
  const u64 unit = wt.units(wt.of(p.key));
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
__device__ int find_token(const Row<F32> &row, uint32_t key, int m, Shared &s) {
  int before = 0;
  for (int base = 0; base < row.n; base += kThreads) {
    const int i = base + threadIdx.x;
    const bool hit = i < row.n && order_key(row.one(i)) == key;
    const u64 b = __ballot(hit);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s.count[threadIdx.x >> 6] = __popcll(b);
    if (threadIdx.x == 0) s.pick[2] = -1;
    __syncthreads();
    int at = before, all = 0;
    for (int w = 0; w < kSampleWaves; ++w) {
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
__device__ void whole_row(const SampleArgs &a, int r, const Row<F32> &row, const Wants &want,
                          const Weights &wt, Shared &s) {
  Place cut = descend(row, wt, s, [&](u64, long long c) { return c >= want.k; });
  if (want.p < 1.0) {
    const double goal = want.p * (double)cut.weight;
    cut = descend(row, wt, s, [&](u64 w, long long) { return (double)w >= goal; });
  }
  u64 total = cut.weight;
  if (wt.of(cut.key) < want.q) {
    // min-p is the shortest run: the weights that reach it
    __syncthreads();
    if (threadIdx.x == 0) s.weight[0] = 0;
    __syncthreads();
    u64 sum = 0;
    row.template each<kThreads>(0, 1, [&](const auto &x, int) {
#pragma unroll 1
      for (int e = 0; e < (int)(sizeof(x) / sizeof(float)); ++e) {
        const double w = wt.of(order_key(x[e]));
        if (w >= want.q) sum += wt.units(w);
      }
    });
    if (sum) atomicAdd(&s.weight[0], sum);
    __syncthreads();
    total = s.weight[0];
  }
  const double goal = want.u * (double)total;
  const Place at = descend(row, wt, s, [&](u64 w, long long) { return (double)w > goal; });
  const int token = find_token(row, at.key, at.m, s);
  if (threadIdx.x == 0) {
    a.token[r] = token;
    if (a.prob) a.prob[r] = (float)(ldexp(wt.of(at.key), a.bits) / (double)total);
  }
}

// ---- by bins ------------------------------------------------------------------

// Sorts n <= kMost distinct tokens of s.token[0] in descending order into
// s.token[1]: 64 at a time within a wavefront, then every token is placed by its
// rank in the other lists of 64.
__device__ __forceinline__ void sort_tokens(int n, Shared &s) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int lists = (n + 63) / 64;
  constexpr int kOwn = kMost / kThreads;       // lists of a wavefront
  u64 x[kOwn];
#pragma unroll
  for (int o = 0; o < kOwn; ++o) {
    const int l = wave + o * kSampleWaves;
    x[o] = l < lists && 64 * l + lane < n ? s.token[0][64 * l + lane] : 0;
    if (l >= lists) continue;
    for (int size = 2; size <= 64; size *= 2)
      for (int gap = size / 2; gap >= 1; gap /= 2) {
        const u64 y = __shfl_xor(x[o], gap, 64);
        const bool first = (lane & gap) == 0, down = (lane & size) == 0;
        x[o] = (x[o] > y) == (first == down) ? x[o] : y;
      }
    (lists == 1 ? s.token[1] : s.token[0])[64 * l + lane] = x[o];
  }
  __syncthreads();
  if (lists == 1) return;
#pragma unroll
  for (int o = 0; o < kOwn; ++o) {
    const int l = wave + o * kSampleWaves;
    if (l >= lists || x[o] == 0) continue;
    int rank = lane;
#pragma unroll 4
    for (int m = 0; m < lists; ++m) {
      const u64 *list = s.token[0] + 64 * m;
      int at = 0;                              // tokens of the list before x
#pragma unroll
      for (int step = 32; step >= 1; step /= 2) at += list[at + step - 1] > x[o] ? step : 0;
      at += list[at] > x[o];
      rank += m == l ? 0 : at;
    }
    s.token[1][rank] = x[o];
  }
  __syncthreads();
}

// Whether the workgroup is to go over the whole row: the bins do not answer.
template <int F32>
__device__ __forceinline__ bool draw_by_bins(const SampleArgs &a, int r, int chunk,
                                             const Row<F32> &row, const Wants &want,
                                             const Ends &ends, const Weights &wt, Shared &s) {
  const float top = wt.top;
  const FastWeights fw = fast_weights(top, ends.low, want.t);
  const u64 *gw = a.weight + (size_t)r * (kBins + 1);
  const int *gc = a.count + (size_t)r * (kBins + 1);
  if (threadIdx.x < kBins / 32) s.wanted[threadIdx.x] = 0;
  if (threadIdx.x == 0) s.pick[0] = 0;
  if (want.k < a.vocab) run_bins<true>(gw, gc, s);
  else run_bins<false>(gw, gc, s);

  // Each filter leaves a weight W; the smallest of the three is drawn from. What
  // the sums of the bins leave open of it, and the bins in which the answers lie
  // (kBins: below 2^-32). Every wavefront finds them by itself.
  auto weight_to = [&](int b) -> u64 { return b < 0 ? 0 : s.weight[min(b, kBins)]; };
  auto reaches = [&](double goal) {
    return min(kBins, first_of(0, kBins + 1, [&](int b) { return (double)s.weight[b] >= goal; }));
  };
  auto exceeds = [&](double goal) {
    return min(kBins, first_of(0, kBins + 1, [&](int b) { return (double)s.weight[b] > goal; }));
  };
  const bool has_k = want.k < a.vocab, has_p = want.p < 1.0, has_q = want.q > 0.0;
  int bk = kBins, p0 = kBins, p1 = kBins, q0 = kBins, q1 = kBins;
  u64 k0 = weight_to(kBins), k1 = k0;
  if (has_k) {
    bk = min(kBins, first_of(0, kBins + 1, [&](int b) { return s.count[b] >= want.k; }));
    k0 = weight_to(bk - 1);
    k1 = weight_to(bk);
    // (below the last bin a token weighs 2^-31.99 at most)
    if (bk == kBins)
      k1 = min(k1, k0 + (u64)(want.k - s.count[kBins - 1]) * ((u64)ldexp(1.01, a.bits - 32) + 1));
  }
  if (has_p) {
    p0 = reaches(want.p * (double)k0);
    p1 = reaches(want.p * (double)k1);
  }
  if (has_q) {
    // the bin of weight q is y below, rounded (its own roundings are far below 0.01)
    const double y = -0.69314718055994530942 / fw.c1 * log2(want.q);
    q0 = y > kBins ? kBins : max(0, (int)rint(y - 0.01));
    q1 = y > kBins ? kBins : min(kBins, (int)rint(y + 0.01));
  }
  const bool cut = has_k || has_p || has_q;
  const int c0 = min(bk, min(p0, q0)), c1 = min(bk, min(p1, q1));
  const int d0 = exceeds(want.u * (double)(cut ? weight_to(c0 - 1) : k0));
  const int d1 = cut ? exceeds(want.u * (double)weight_to(c1)) : d0;
  const bool get_k = bk < kBins && (has_p || bk <= c1);
  const int pe = min(p1, min(c1, kBins - 1)), qe = min(q1, min(c1, kBins - 1));
  if (d1 >= kBins) {                           // a draw from below 2^-32
    return chunk == 0;
  }
  // Those bins, and bounds on the logits in them (rounded outwards): nearly every
  // token is left by the bounds, two comparisons for each of the bounds there are.
  float low[4], high[4];
  int bounds = 0;
  auto want_bins = [&](bool any, int b0, int b1) {
    if (!any) return;
    const float d1 = (float)((b1 + 0.51) / fw.slope), d0 = (float)((b0 - 0.51) / fw.slope);
    const float lo = top - d1 - 1e-5f * (__builtin_fabsf(top) + d1);
    const float hi = top - d0 + 1e-5f * (__builtin_fabsf(top) + __builtin_fabsf(d0));
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i == bounds) {
        low[i] = lo;
        high[i] = hi;
      }
    ++bounds;
    for (int b = b0 + (int)threadIdx.x; b <= b1; b += kThreads)
      atomicOr(&s.wanted[b >> 5], 1u << (b & 31));
  };
  want_bins(true, d0, d1);
  want_bins(get_k, bk, bk);
  want_bins(has_p && p0 <= pe, p0, pe);
  want_bins(has_q && q0 <= qe, q0, qe);
  __syncthreads();
  auto collect = [&](auto bounds_there) {
    constexpr int B = decltype(bounds_there)::value;
    row.template each<kThreads>(chunk, a.draws, [&](const auto &x, int i) {
      constexpr int N = sizeof(x) / sizeof(float);
      bool hit[N], any = false;
#pragma unroll
      for (int e = 0; e < N; ++e) {
        hit[e] = x[e] >= low[0] && x[e] <= high[0];
#pragma unroll
        for (int j = 1; j < B; ++j) hit[e] |= x[e] >= low[j] && x[e] <= high[j];
        any |= hit[e];
      }
      if (!any) return;
      uint32_t hits = 0;                       // one each time, of a lane that has several
#pragma unroll
      for (int e = 0; e < N; ++e) hits |= hit[e] ? 1u << e : 0u;
      do {
        const int at_e = __builtin_ctz(hits);
        hits &= hits - 1;
        float v = x[0];
#pragma unroll
        for (int e = 1; e < N; ++e) v = at_e == e ? x[e] : v;
        const int b = fw.bin_of(v);
        if (b >= 0 && b < kBins && (s.wanted[b >> 5] >> (b & 31) & 1)) {
          const int at = atomicAdd(&s.pick[0], 1);
          if (at < kMost) s.token[0][at] = token_of(order_key(v), i + at_e);
        }
      } while (hits);
    });
  };
  if (bounds == 1) collect(std::integral_constant<int, 1>{});
  else if (bounds == 2) collect(std::integral_constant<int, 2>{});
  else {
    if (bounds == 3) {
      low[3] = low[2];
      high[3] = high[2];
    }
    collect(std::integral_constant<int, 4>{});
  }
  __syncthreads();
  int n = s.pick[0];
  if (a.draws > 1) {
    // collected so far in the lower 20 bits of the row's state (a workgroup adds
    // kMost + 1 at most), workgroups done above
    constexpr int kDone = 1 << 20;
    u64 *list = a.list + (size_t)r * kMost;
    if (n) {
      if (threadIdx.x == 0)
        s.pick[1] = __hip_atomic_fetch_add(a.state + r, min(n, kMost + 1), __ATOMIC_RELAXED,
                                           __HIP_MEMORY_SCOPE_AGENT) & (kDone - 1);
      __syncthreads();
      const int at = s.pick[1];
      for (int i = threadIdx.x; i < min(n, kMost); i += kThreads)
        if (at + i < kMost)
          __hip_atomic_store(list + at + i, s.token[0][i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0F70);        // vmcnt(0): this wave's stores are complete
    asm volatile("" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0)
      s.pick[1] = __hip_atomic_fetch_add(a.state + r, kDone, __ATOMIC_RELAXED,
                                         __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    if (s.pick[1] / kDone != a.draws - 1) return false;
    n = s.pick[1] & (kDone - 1);
    if (n <= kMost)
      for (int i = threadIdx.x; i < n; i += kThreads)
        s.token[0][i] = __hip_atomic_load(list + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
  }
  if (n > kMost) return true;
  sort_tokens(n, s);
  const u64 *token = s.token[1];
  u64 *sum = s.token[0];
  auto value_at = [&](int i) { return key_value((uint32_t)(token[i] >> 32)); };
  for (int i = threadIdx.x; i < n; i += kThreads) {
    const float x = value_at(i);
    const double z = fw.below(x), t = fw.nearest(z);
    const int b = FastWeights::bin(t);
    sum[i] = fw.units(z, t, b, fw.unit_of(b, a.bits));
    if (i == 0 || fw.bin_of(value_at(i - 1)) != b) s.start[b] = (uint16_t)i;
    if (i == n - 1 || fw.bin_of(value_at(i + 1)) != b) s.stop[b] = (uint16_t)(i + 1);
  }
  __syncthreads();
  run_sums(sum, n, s);
  // running weight up to and with sorted token i of bin b, whose tokens start at i0
  auto weight_at = [&](int i, int b, int i0) -> u64 {
    return weight_to(b - 1) + sum[i] - (i0 > 0 ? sum[i0 - 1] : 0);
  };
  // the first sorted token of bin b whose running weight passes, and that weight
  auto place = [&](int b, u64 &weight, auto passes) {
    const int i0 = min((int)s.start[b], n - 1), i1 = min((int)s.stop[b], n);
    const int i = min(first_of(i0, i1, [&](int j) { return passes(weight_at(j, b, i0)); }),
                      max(i0, i1 - 1));
    weight = weight_at(i, b, i0);
    return i;
  };
  // false: the bins do not answer
  auto answer = [&]() {
    u64 w0 = k0, w1 = k1;
    if (get_k) {
      const int i0 = min((int)s.start[bk], n - 1);
      const int i = min(n - 1, i0 + want.k - (bk > 0 ? s.count[bk - 1] : 0) - 1);
      w0 = w1 = weight_at(i, bk, i0);
    }
    if (has_p) {
      auto run = [&](double goal, u64 least) {
        const int b = reaches(goal);
        u64 w = b < kBins ? weight_to(b) : least;
        if (b <= pe) place(b, w, [&](u64 x) { return (double)x >= goal; });
        return w;
      };
      const u64 p_low = run(want.p * (double)w0, weight_to(kBins - 1));
      const u64 p_high = w0 == w1 && p1 < kBins ? p_low : run(want.p * (double)w1, weight_to(kBins));
      w0 = min(w0, p_low);
      w1 = min(w1, p_high);
    }
    if (has_q) {
      // the first token of the bins around q that does not reach it
      const int i = first_of(0, n, [&](int j) {
        const int b = fw.bin_of(value_at(j));
        return b > qe || (b >= q0 && wt.of((uint32_t)(token[j] >> 32)) < want.q);
      });
      const int b = i < n ? fw.bin_of(value_at(i)) : kBins;
      if (b <= qe) {
        const int i0 = min((int)s.start[b], n - 1);
        const u64 w = i > i0 ? weight_at(i - 1, b, i0) : weight_to(b - 1);
        w0 = min(w0, w);
        w1 = min(w1, w);
      } else {
        w0 = min(w0, weight_to(qe));
        w1 = min(w1, weight_to(q1 < kBins ? qe : kBins));
      }
    }
    auto draw = [&](u64 total) {
      const double goal = want.u * (double)total;
      u64 w;
      return place(exceeds(goal), w, [&](u64 x) { return (double)x > goal; });
    };
    // What lies below 2^-32 may leave the weight open: not if it does not matter (the
    // probability is then off by 2^-25, and by 2^-24 for its rounding).
    const int i = draw(w0);
    if (w0 != w1 && ((double)(w1 - w0) > 0x1p-24 * (double)w0 || draw(w1) != i)) return false;
    if (threadIdx.x == 0) {
      a.token[r] = index_of(token[i]);
      if (a.prob)
        a.prob[r] = (float)(ldexp(wt.of((uint32_t)(token[i] >> 32)), a.bits) / (0.5 * ((double)w0 + (double)w1)));
    }
    return true;
  };
  if (threadIdx.x < 64) {
    const bool answered = answer();
    if (threadIdx.x == 0) s.pick[2] = !answered;
  }
  __syncthreads();
  return s.pick[2] != 0;
}

template <int F32>
__global__ __launch_bounds__(kThreads) void sample_draw_kernel(SampleArgs a) {
  __shared__ Shared s;
  const int chunk = blockIdx.x, r = blockIdx.y;
  const Row<F32> row(a, r);
  const Wants want = wants_of(a, r);
  const Ends ends = row_ends(a, r);
  const uint32_t top = (uint32_t)(ends.best >> 32);
  if (top == 0 || !drawn(want)) {               // nothing above -inf, or no draw
    if (chunk == 0 && threadIdx.x == 0) {
      a.token[r] = top == 0 ? -1 : index_of(ends.best);
      if (a.prob) a.prob[r] = top == 0 ? 0.f : 1.f;
    }
    return;
  }
  // (not 0 at an infinite temperature, at which only tokens of +inf weigh where there are any)
  const Weights wt{key_value(top), fmax(1.4426950408889634074 / (double)want.t, 1e-300), a.bits};
  const bool whole =
      by_bins(want, top) ? draw_by_bins(a, r, chunk, row, want, ends, wt, s) : chunk == 0;
  if (whole) whole_row(a, r, row, want, wt, s);
}

template <int F32>
void launch(const SampleArgs &a, hipStream_t s) {
  const dim3 grid((unsigned)a.chunks, (unsigned)a.rows);
  hipLaunchKernelGGL(sample_top_kernel<F32>, grid, dim3(kSumThreads), 0, s, a);
  hipLaunchKernelGGL(sample_bins_kernel<F32>, grid, dim3(kSumThreads), 0, s, a);
  hipLaunchKernelGGL(sample_draw_kernel<F32>, dim3((unsigned)a.draws, (unsigned)a.rows),
                     dim3(kThreads), 0, s, a);
}

}  // namespace

// Workspace: [tops][lows][weights][counts][lists][states].
SampleLayout sample_layout(int rows, int vocab, int cus) {
  SampleLayout l;
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  // Chunks of at least a load per thread (of bf16 logits): about two workgroups per
  // CU for the sums, or four where they have 16K tokens each (64 x 151936: 18 us
  // with two, 21 with four, whose bins are twice as many to add up; 320 x 151937:
  // 50 with four, 68 with two); one for the draws.
  const int most = std::max(1, vocab / (8 * kSumThreads));
  l.chunks = std::max(1, std::min(most, std::max(2 * cus / rows,
                                                 std::min(4 * cus / rows, vocab / 16384))));
  l.draws = std::max(1, std::min(std::max(1, vocab / (8 * kThreads)), cus / rows));
  const size_t n = (size_t)rows;
  l.lows = up(n * l.chunks * sizeof(u64));
  l.weight = l.lows + up(n * l.chunks * sizeof(float));
  l.count = l.weight + up(n * (kBins + 1) * sizeof(u64));
  l.list = l.count + up(n * (kBins + 1) * sizeof(int32_t));
  l.state = l.list + up(n * kMost * sizeof(u64));
  l.total = l.state + up(n * sizeof(int32_t));
  return l;
}

hipError_t launch_sample(const SampleArgs &a, hipStream_t s) {
  if (a.f32) launch<1>(a, s);
  else launch<0>(a, s);
  return hipGetLastError();
}

}  // namespace kap

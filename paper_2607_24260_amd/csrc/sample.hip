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
//   1  the largest logit of every chunk;
//   2  a histogram of weights and counts over bins of 2^(1/32) of weight below
//      the largest, down to 2^-32 (one bin for all that is less);
//   3  from the running sums of the bins, those that an answer can lie in; their
//      tokens are collected, and the last workgroup of the row sorts them and
//      finds the answers among them.
// Rows for which that is not few tokens (thousands of equal logits, a top-k or
// draw among weights below 2^-32) are descended eight bits of the logit at a
// time over the whole row instead, by the same last workgroup.
//
// The weights are summed as integers, in units of 2^-s with s = 62 - ceil(log2
// vocab): the sums do not depend on their order, and a running weight is off by
// less than vocab half units, where 32-bit floats would move the boundaries
// between tokens by as much as whole tokens.
#include "kap_internal.h"

#include <algorithm>

namespace kap {
namespace {

constexpr int kThreads = 512;
constexpr int kSampleWaves = kThreads / 64;
// Bins: kPerOctave per factor of two in weight, kOctaves of them.
constexpr int kPerOctave = 32;
constexpr int kBins = 1024;
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
  // f(logit, index) for every token of a chunk, a thread's tokens in ascending order
  template <class F>
  __device__ void each(int chunk, int chunks, F f) const {
    if (chunk == 0 && (int)threadIdx.x < head) f(one(threadIdx.x), (int)threadIdx.x);
    const kv_u32x4 *v = reinterpret_cast<const kv_u32x4 *>(x + (size_t)head * (F32 ? 4 : 2));
    const int per = (vecs + chunks - 1) / chunks;
    const int v0 = chunk * per, v1 = min(vecs, v0 + per);
    auto use = [&](const kv_u32x4 &w, int j) {
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        const float y = F32 ? __uint_as_float(w[e & 3])
                            : ((e & 1) ? bf16_hi(w[(e >> 1) & 3]) : bf16_lo(w[(e >> 1) & 3]));
        f(y, head + j * kVec + e);
      }
    };
    int j = v0 + threadIdx.x;
    for (; j + kThreads < v1; j += 2 * kThreads) {
      const kv_u32x4 w0 = v[j], w1 = v[j + kThreads];
      use(w0, j);
      use(w1, j + kThreads);
    }
    if (j < v1) use(v[j], j);
    if (chunk == chunks - 1) {
      const int i = head + vecs * kVec + (int)threadIdx.x;
      if (i < n) f(one(i), i);
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

// The same to 2^-48 of a weight, and its bin, for the sums over whole rows: with
// y = 32 log2 w, n = rint(y): 2^(n / 32) from a table of 32 and 2^((y - n) / 32)
// by its series to the fifth power ((ln 2 / 64)^6 / 6! = 2^-48.7).
struct FastWeights {
  double slope, offset;                        // y = x * slope + offset
  double unit;                                 // 2^bits
  const double *table;                         // 2^(i / 32), in LDS
  __device__ static constexpr double magic() { return 6755399441055744.0; }   // 1.5 * 2^52
  __device__ double shifted(float x) const { return fma((double)x, slope, offset) + magic(); }
  // whether a logit has a bin (NaN and -inf have none)
  __device__ static bool binned(double t) { return t > magic() - kBins; }
  __device__ static int bin(double t) { return -(int)(uint32_t)__double_as_longlong(t); }
  __device__ u64 units(float x, double t) const {
    constexpr double c = 0.69314718055994530942 / 32;
    const int n = (int)(uint32_t)__double_as_longlong(t);
    const double f = fma((double)x, slope, offset) - (t - magic());
    const double p =
        f * (c + f * (c * c / 2 + f * (c * c * c / 6 +
                                       f * (c * c * c * c / 24 + f * (c * c * c * c * c / 120)))));
    const double s = table[n & 31];
    const double w = ldexp(fma(s, p, s), n >> 5);
    return (u64)__double_as_longlong(fma(w, unit, 4503599627370496.0)) & 0xfffffffffffffull;
  }
};

__device__ __forceinline__ FastWeights fast_weights(float top, float t, int bits, double *table) {
  if (threadIdx.x < 32) table[threadIdx.x] = exp2(threadIdx.x / 32.0);
  const double slope = 32 * 1.4426950408889634074 / (double)t;
  return FastWeights{slope, -(double)top * slope, ldexp(1.0, bits), table};
}

// What a row asks for.
struct Wants {
  bool greedy;
  int k;             // vocab: no top-k
  double p, q, u;    // p 1: no top-p; q 0: no min-p
};
__device__ __forceinline__ Wants wants_of(const SampleArgs &a, int r) {
  Wants w;
  const float t = a.temperature ? a.temperature[r] : 1.f;
  w.greedy = !(t > 0.f);
  w.k = a.top_k && a.top_k[r] > 0 ? min(a.top_k[r], a.vocab) : a.vocab;
  w.p = a.top_p && a.top_p[r] < 1.f ? (double)a.top_p[r] : 1.0;
  w.q = a.min_p && a.min_p[r] > 0.f ? fmin((double)a.min_p[r], 1.0) : 0.0;
  const double u = a.uniform[r];
  w.u = u > 0.0 ? fmin(u, 1.0 - 0x1p-24) : 0.0;
  return w;
}

// The largest token of a row from its chunks' (every wavefront by itself).
__device__ __forceinline__ u64 row_top(const SampleArgs &a, int r) {
  u64 best = 0;
  for (int c = threadIdx.x & 63; c < a.chunks; c += 64) best = max(best, a.tops[(size_t)r * a.chunks + c]);
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) best = max(best, __shfl_xor(best, o, 64));
  return best;
}

// Whether the histogram serves a row: a drawn one whose largest logit and
// temperature give finite coefficients.
__device__ __forceinline__ bool by_bins(const Wants &w, uint32_t top, float t) {
  return !w.greedy && key_value(top) < INFINITY && t > 1e-30f;
}

// ---------------------------------------------------------------------------
// 1: the largest logit of every chunk; the row's sums are cleared
// ---------------------------------------------------------------------------

template <int F32>
__global__ __launch_bounds__(kThreads) void sample_top_kernel(SampleArgs a) {
  __shared__ u64 s_best[kSampleWaves];
  const int chunk = blockIdx.x, r = blockIdx.y;
  const Row<F32> row(a, r);
  float best = -INFINITY;
  int at = -1;
  row.each(chunk, a.chunks, [&](float x, int i) {
    if (x > best) {
      best = x;
      at = i;
    }
  });
  u64 token = at < 0 ? 0 : token_of(order_key(best), at);
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) token = max(token, __shfl_xor(token, o, 64));
  if ((threadIdx.x & 63) == 0) s_best[threadIdx.x >> 6] = token;
  for (int i = chunk * kThreads + threadIdx.x; i <= kBins; i += a.chunks * kThreads) {
    a.weight[(size_t)r * (kBins + 1) + i] = 0;
    a.count[(size_t)r * (kBins + 1) + i] = 0;
  }
  if (chunk == 0 && threadIdx.x < 2) a.state[2 * r + threadIdx.x] = 0;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < kSampleWaves; ++w) token = max(token, s_best[w]);
    a.tops[(size_t)r * a.chunks + chunk] = token;
  }
}

// ---------------------------------------------------------------------------
// 2: weights and counts by bin
// ---------------------------------------------------------------------------

template <int F32>
__global__ __launch_bounds__(kThreads) void sample_bins_kernel(SampleArgs a) {
  __shared__ u64 s_weight[kBins + 1];
  __shared__ int s_count[kBins + 1];
  __shared__ double s_table[32];
  const int chunk = blockIdx.x, r = blockIdx.y;
  const Wants want = wants_of(a, r);
  const uint32_t top = (uint32_t)(row_top(a, r) >> 32);
  const float t = a.temperature ? a.temperature[r] : 1.f;
  if (top == 0 || !by_bins(want, top, t)) return;
  const FastWeights w = fast_weights(key_value(top), t, a.bits, s_table);
  for (int i = threadIdx.x; i <= kBins; i += kThreads) {
    s_weight[i] = 0;
    s_count[i] = 0;
  }
  __syncthreads();
  const bool counts = want.k < a.vocab;
  u64 rest = 0;
  int rest_n = 0;
  const Row<F32> row(a, r);
  row.each(chunk, a.chunks, [&](float x, int) {
    const double s = w.shifted(x);
    const int b = FastWeights::bin(s);
    if (FastWeights::binned(s)) {
      atomicAdd(&s_weight[b], w.units(x, s));
      if (counts) atomicAdd(&s_count[b], 1);
    } else {
      // below 2^-32: 32-bit exponentials are exact to 2^-55
      const float y = (float)fma((double)x, w.slope, w.offset) * (1.f / kPerOctave);
      const float e = exp2f(y);
      rest += e > 0.f ? (u64)(e * (float)w.unit) : 0;
      ++rest_n;
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
  for (int i = threadIdx.x; i <= kBins; i += kThreads) {
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
  u64 token[kMost];                            // sorted: descending
  u64 sum[kMost];                              // running units of the sorted tokens
  uint32_t wanted[kBins / 32];
  u64 red[kSampleWaves];
  double table[32];
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

// Inclusive running sums over n values of LDS, in place.
template <typename T>
__device__ void run_sums(T *x, int n, Shared &s) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  u64 before = 0;
  for (int base = 0; base < n; base += kThreads) {
    const int i = base + threadIdx.x;
    T v = i < n ? x[i] : T(0);
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const T y = __shfl_up(v, o, 64);
      if (lane >= o) v += y;
    }
    __syncthreads();
    if (lane == 63) s.red[wave] = (u64)v;
    __syncthreads();
    u64 add = before, all = 0;
    for (int w = 0; w < kSampleWaves; ++w) {
      if (w < wave) add += s.red[w];
      all += s.red[w];
    }
    if (i < n) x[i] = v + (T)add;
    before += all;
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
    row.each(0, 1, [&](float x, int) {
      const uint32_t k = order_key(x);
      if (shift < 24 && (k >> (shift + 8)) != (p.key >> (shift + 8))) return;
      const int bin = (k >> shift) & (kDigits - 1);
      atomicAdd(&s.count[bin], 1);
      atomicAdd(&s.weight[bin], wt.units(wt.of(k)));
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
    row.each(0, 1, [&](float x, int) {
      const double w = wt.of(order_key(x));
      if (w >= want.q) sum += wt.units(w);
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

// Sorts n tokens of LDS in descending order (n rounded up to a power of two).
__device__ void sort_tokens(u64 *x, int n) {
  int m = 2;
  while (m < n) m *= 2;
  for (int i = n + threadIdx.x; i < m; i += kThreads) x[i] = 0;
  __syncthreads();
  for (int size = 2; size <= m; size *= 2)
    for (int gap = size / 2; gap >= 1; gap /= 2) {
      for (int i = threadIdx.x; i < m / 2; i += kThreads) {
        const int lo = 2 * i - (i & (gap - 1)), hi = lo + gap;
        const u64 p = x[lo], q = x[hi];
        if ((p < q) == ((lo & size) == 0)) {
          x[lo] = q;
          x[hi] = p;
        }
      }
      __syncthreads();
    }
}

// Whether the workgroup is to go over the whole row: the bins do not answer.
template <int F32>
__device__ __forceinline__ bool draw_by_bins(const SampleArgs &a, int r, int chunk,
                                             const Row<F32> &row, const Wants &want, uint32_t top,
                                             float t, const Weights &wt, Shared &s) {
  const FastWeights fw = fast_weights(key_value(top), t, a.bits, s.table);
  const u64 *gw = a.weight + (size_t)r * (kBins + 1);
  const int *gc = a.count + (size_t)r * (kBins + 1);
  for (int i = threadIdx.x; i <= kBins; i += kThreads) {
    s.weight[i] = gw[i];
    s.count[i] = gc[i];
  }
  if (threadIdx.x < kBins / 32) s.wanted[threadIdx.x] = 0;
  __syncthreads();
  run_sums(s.weight, kBins + 1, s);
  if (want.k < a.vocab) run_sums(s.count, kBins + 1, s);

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
  }
  if (has_p) {
    p0 = reaches(want.p * (double)k0);
    p1 = reaches(want.p * (double)k1);
  }
  if (has_q) {
    // the bin of weight q is -32 log2 q, rounded; its neighbours cover the roundings
    const double y = -kPerOctave * log2(want.q);
    q0 = y > kBins ? kBins : max(0, (int)y - 1);
    q1 = min(kBins, q0 + 3);
  }
  const bool cut = has_k || has_p || has_q;
  const int c0 = min(bk, min(p0, q0)), c1 = min(bk, min(p1, q1));
  const int d0 = exceeds(want.u * (double)(cut ? weight_to(c0 - 1) : k0));
  const int d1 = cut ? exceeds(want.u * (double)weight_to(c1)) : d0;
  const bool get_k = bk < kBins && (has_p || bk <= c1);
  const int pe = min(p1, min(c1, kBins - 1)), qe = min(q1, min(c1, kBins - 1));
  const int last = max(max(get_k ? bk : 0, d1), max(has_p ? pe : 0, has_q ? qe : 0));
  if (d1 >= kBins) {                           // a draw from below 2^-32
    return chunk == 0;
  }
  auto want_bins = [&](int b0, int b1) {
    for (int b = b0 + (int)threadIdx.x; b <= b1; b += kThreads)
      atomicOr(&s.wanted[b >> 5], 1u << (b & 31));
  };
  if (get_k) want_bins(bk, bk);
  if (has_p) want_bins(p0, pe);
  if (has_q) want_bins(q0, qe);
  want_bins(d0, d1);

  // The tokens of those bins. (A logit below `least` is in none of them.)
  const float least =
      key_value(top) - (float)((last + 2) * (double)t / (kPerOctave * 1.4426950408889634074)) * 1.0001f -
      1e-5f * __builtin_fabsf(key_value(top));
  if (threadIdx.x == 0) s.pick[0] = 0;
  __syncthreads();
  row.each(chunk, a.chunks, [&](float x, int i) {
    if (!(x >= least)) return;
    const double sh = fw.shifted(x);
    const int b = FastWeights::bin(sh);
    if (!FastWeights::binned(sh) || b > last || !(s.wanted[b >> 5] >> (b & 31) & 1)) return;
    const int at = atomicAdd(&s.pick[0], 1);
    if (at < kMost) s.token[at] = token_of(order_key(x), i);
  });
  __syncthreads();
  const int mine = s.pick[0];
  u64 *list = a.list + (size_t)r * kMost;
  if (a.chunks > 1) {
    int *state = a.state + 2 * r;              // tokens collected, workgroups done
    if (threadIdx.x == 0 && mine)
      s.pick[1] = __hip_atomic_fetch_add(state, mine, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    if (mine) {
      const int at = s.pick[1];
      for (int i = threadIdx.x; i < mine; i += kThreads)
        if (i < kMost && at + i < kMost)
          __hip_atomic_store(list + at + i, s.token[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    if (!last_arrival_of(state + 1, a.chunks, &s.pick[3])) return false;
    if (threadIdx.x == 0)
      s.pick[0] = __hip_atomic_load(state, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
  }
  const int n = s.pick[0];
  if (n > kMost) {
    return true;
  }
  if (a.chunks > 1)
    for (int i = threadIdx.x; i < n; i += kThreads)
      s.token[i] = __hip_atomic_load(list + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  sort_tokens(s.token, n);
  auto value_at = [&](int i) { return key_value((uint32_t)(s.token[i] >> 32)); };
  auto bin_at = [&](int i) { return FastWeights::bin(fw.shifted(value_at(i))); };
  for (int i = threadIdx.x; i < n; i += kThreads) s.sum[i] = fw.units(value_at(i), fw.shifted(value_at(i)));
  __syncthreads();
  run_sums(s.sum, n, s);

  // running weight up to and with sorted token i of bin b, whose tokens start at i0
  auto start_of = [&](int b) { return first_of(0, n, [&](int i) { return bin_at(i) >= b; }); };
  auto weight_at = [&](int i, int b, int i0) -> u64 {
    return weight_to(b - 1) + s.sum[i] - (i0 > 0 ? s.sum[i0 - 1] : 0);
  };
  // the first sorted token of bin b whose running weight passes, and that weight
  auto place = [&](int b, u64 &weight, auto passes) {
    const int i0 = start_of(b), i1 = start_of(b + 1);
    const int i = min(first_of(i0, i1, [&](int j) { return passes(weight_at(j, b, i0)); }),
                      max(i0, i1 - 1));
    weight = weight_at(i, b, i0);
    return i;
  };
  if (get_k) {
    const int i0 = start_of(bk);
    const int i = min(n - 1, i0 + want.k - (bk > 0 ? s.count[bk - 1] : 0) - 1);
    k0 = k1 = weight_at(i, bk, i0);
  }
  u64 w0 = k0, w1 = k1;
  if (has_p) {
    auto run = [&](double goal, u64 least) {
      const int b = reaches(goal);
      u64 w = b < kBins ? weight_to(b) : least;
      if (b <= pe) place(b, w, [&](u64 x) { return (double)x >= goal; });
      return w;
    };
    w0 = min(w0, run(want.p * (double)k0, weight_to(kBins - 1)));
    w1 = min(w1, run(want.p * (double)k1, weight_to(kBins)));
  }
  if (has_q) {
    const int i0 = start_of(q0), i1 = start_of(qe + 1);
    const int i = first_of(i0, i1, [&](int j) { return wt.of((uint32_t)(s.token[j] >> 32)) < want.q; });
    if (i < i1) {
      const int b = bin_at(i), ib = start_of(b);
      const u64 w = i > ib ? weight_at(i - 1, b, ib) : weight_to(b - 1);
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
  // What lies below 2^-32 may leave the weight open: not if it does not matter.
  const int i = draw(w0);
  if (w0 != w1 && ((double)(w1 - w0) > 0x1p-26 * (double)w0 || draw(w1) != i)) {
    return true;
  }
  if (threadIdx.x == 0) {
    const u64 token = s.token[i];
    a.token[r] = index_of(token);
    if (a.prob) a.prob[r] = (float)(ldexp(wt.of((uint32_t)(token >> 32)), a.bits) / (double)w1);
  }
  return false;
}

template <int F32>
__global__ __launch_bounds__(kThreads) void sample_draw_kernel(SampleArgs a) {
  __shared__ Shared s;
  const int chunk = blockIdx.x, r = blockIdx.y;
  const Row<F32> row(a, r);
  const Wants want = wants_of(a, r);
  const u64 best = row_top(a, r);
  const uint32_t top = (uint32_t)(best >> 32);
  const float t = a.temperature ? a.temperature[r] : 1.f;
  if (top == 0 || want.greedy) {               // nothing above -inf, or no draw
    if (chunk == 0 && threadIdx.x == 0) {
      a.token[r] = top == 0 ? -1 : index_of(best);
      if (a.prob) a.prob[r] = top == 0 ? 0.f : 1.f;
    }
    return;
  }
  const Weights wt{key_value(top), 1.4426950408889634074 / (double)t, a.bits};
  const bool whole = by_bins(want, top, t) ? draw_by_bins(a, r, chunk, row, want, top, t, wt, s)
                                           : chunk == 0;
  if (whole) whole_row(a, r, row, want, wt, s);
}

template <int F32>
void launch(const SampleArgs &a, hipStream_t s) {
  const dim3 grid((unsigned)a.chunks, (unsigned)a.rows);
  hipLaunchKernelGGL(sample_top_kernel<F32>, grid, dim3(kThreads), 0, s, a);
  hipLaunchKernelGGL(sample_bins_kernel<F32>, grid, dim3(kThreads), 0, s, a);
  hipLaunchKernelGGL(sample_draw_kernel<F32>, grid, dim3(kThreads), 0, s, a);
}

}  // namespace

// Workspace: [tops][weights][counts][lists][states].
SampleLayout sample_layout(int rows, int vocab, int cus) {
  SampleLayout l;
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  // about two workgroups per CU, of at least a load per thread (of bf16 logits)
  const int most = std::max(1, vocab / (8 * kThreads));
  l.chunks = std::max(1, std::min(most, 2 * cus / rows));
  const size_t n = (size_t)rows;
  l.weight = up(n * l.chunks * sizeof(u64));
  l.count = l.weight + up(n * (kBins + 1) * sizeof(u64));
  l.list = l.count + up(n * (kBins + 1) * sizeof(int32_t));
  l.state = l.list + up(n * kMost * sizeof(u64));
  l.total = l.state + up(n * 2 * sizeof(int32_t));
  return l;
}

hipError_t launch_sample(const SampleArgs &a, hipStream_t s) {
  if (a.f32) launch<1>(a, s);
  else launch<0>(a, s);
  return hipGetLastError();
}

}  // namespace kap

// Verification and decode attention of sequences that share leading pages
// (groups of requests over one document): the shared pages are walked once with
// the query rows of all the group's sequences, then every sequence's own pages
// with its own rows, and the parts are merged by their log-sum-exp.
//
// A unit is (rows, pages): a group's rows over its shared pages, or a sequence's
// q_len * G rows over its own. A wavefront holds 32 rows and walks 32 keys (two
// pages) a step:
//   S^T[key][row] = K . Q^T       v_mfma_f32_32x32x16_bf16, or
//   O^T[dim][row] += V^T P^T      v_mfma_f32_32x32x2_f32 for float32 KV
// The accumulator of S^T gives lane l row l % 32 and 16 of the keys, the other
// lane of that row the rest; with the keys of K's operand in the order of
// key_of_row() those are eight neighbouring keys of either page, which is the
// layout P^T's operand needs: weights never leave their lane.
//
// A workgroup takes 32 rows of a group and a split of its shared pages, a step for
// each of its wavefronts in turn; a wavefront by itself takes up to 32 rows of a
// sequence and a split of its own pages. Operands go straight from memory (or, where
// other rows read the same pages, the caches) to the lane's registers, the next
// step's on the way while this one is multiplied, and no wavefront waits for another
// before the end: the matrix instructions of one then fall into the vector
// instructions of the other. (Pages shared out through LDS, read once by wavefronts
// with up to 256 rows between them, took 88 us where this takes 90 for 256 rows over
// 32K positions, bf16 and 128 dims, but 56 us where this takes 53 for 128 rows, 56
// and 45 with fp8 pages, 62 and 48 with 64 dims: barriers, and rows rounded up to a
// power of two.)
//
// Weights are float32. For 16-bit V they are split into three bf16 parts, each
// rounded to nearest: what is left out is at most 2^-27 of a weight, so that outputs
// are good to single precision (off by 3e-7 to 7e-7 of their norm; with two parts,
// 2^-18, by 2.4e-6, for 94 instead of 97 us at 64 x 32K and 257 instead of 292 us for
// four groups of 80 rows with fp8 pages). The reference they are taken against
// stays above every logit: when one exceeds it, it moves kDefer beyond (in powers
// of two), so that it hardly ever moves and no weight exceeds 1.
//
// Measured (128 dims, 8 KV heads, 32 query heads): 8 sequences over 16K shared
// positions, bf16 (76 MB) 27.1 us: the walk itself is 9 us, as fast as the bytes come
// from the caches, and around it the launches, the work map (2), the first loads (3),
// the workgroup's sum over its wavefronts (3) and the merge's launch (5). 64 over 32K
// (256 rows a KV head; 35 GFLOP, of which those with V are done for each part) 97 to
// 100 us: matrix and vector instructions of two wavefronts per SIMD. Four groups of four
// over 32K to 128K, 5-token windows, fp8 (80 rows, 670 MB) 294 to 306 us: the same, with
// 96 rows multiplied for 80. Two sequences over 1000 positions, float32, 64 dims 21 us:
// the chain of launches, map, two steps a wavefront and merge.
#include "kap_internal.h"

#include <algorithm>
#include <type_traits>

namespace kap {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kRows = 32;                      // of a wavefront
constexpr int kKeys = 32;                      // of a step
// Wavefronts of a workgroup: two per SIMD, or one where accumulators, queries and
// a step's operands leave no room for a second.
constexpr int waves_of(int kv, int D) { return D == 256 || (kv == kF32 && D == 128) ? 4 : 8; }

__device__ __forceinline__ f32x16 mfma(u32x4 a, u32x4 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a),
                                                 __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mfma(float a, float b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 zero16() {
  f32x16 z;
#pragma unroll
  for (int i = 0; i < 16; ++i) z[i] = 0.f;
  return z;
}

// x of the lane that has the same row (32 lanes on).
__device__ __forceinline__ float other_half(float x) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_int(x), __float_as_int(x), false, false);
  return __int_as_float((threadIdx.x & 32) ? r[0] : r[1]);
}

// Key (0..31, of two pages) in row i of K's operand, and the in-page key of
// accumulator register r (page r / 8) in half hb of the wavefront.
template <int KV>
__device__ __forceinline__ int key_of_row(int i) {
  return KV == kF32 ? i : (i & 19) | (i & 4) << 1 | (i & 8) >> 1;
}
template <int KV>
__device__ __forceinline__ int key_of_reg(int r, int hb) {
  return KV == kF32 ? (r & 3) + 8 * (r >> 2 & 1) + 4 * hb : 8 * hb + (r & 7);
}

constexpr int elem_bytes(int kv) { return kv == kF32 ? 4 : (kv == kBF16 ? 2 : 1); }

// ---------------------------------------------------------------------------
// work map
// ---------------------------------------------------------------------------

struct Item {
  bool shared;       // a group's shared pages, or a sequence's own
  int seq0, rows;    // first sequence and rows of the unit
  int page0, pages;  // pages of the unit, in table row seq0
  int rb, g, split, n_split;
  int64_t row0;      // partial rows of the unit start here
  int unit;          // group or sequence
};

struct Unit {
  int seq0, rows, page0, pages;
};

__device__ __forceinline__ int clamp_to(int x, int lo, int hi) { return min(max(x, lo), hi); }

__device__ __forceinline__ Unit group_unit(const SharedArgs &a, int g) {
  const int o0 = clamp_to(a.offsets[g], 0, a.batch), o1 = clamp_to(a.offsets[g + 1], o0, a.batch);
  return Unit{o0, (o1 - o0) * a.q_len * a.G, 0, o1 > o0 ? clamp_to(a.shared[g], 0, a.max_pages) : 0};
}

// The group that holds sequence b, or -1.
__device__ __forceinline__ int group_of(const SharedArgs &a, int b) {
  int lo = 0, hi = a.num_groups;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (a.offsets[mid] <= b) lo = mid;
    else hi = mid;
  }
  return a.num_groups > 0 && a.offsets[lo] <= b && b < a.offsets[lo + 1] ? lo : -1;
}

__device__ __forceinline__ Unit seq_unit(const SharedArgs &a, int b) {
  const int g = group_of(a, b);
  const int L = a.seq_lens[b];
  const int np = L > 0 ? min((int)(((long long)L + kPage - 1) / kPage), a.max_pages) : 0;
  const int sh = g >= 0 ? clamp_to(a.shared[g], 0, a.max_pages) : 0;
  return Unit{b, a.q_len * a.G, sh, max(0, np - sh)};
}

__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) x += __shfl_xor(x, o, 64);
  return x;
}

// Work item of a wavefront. C steps are what a workgroup gets; shared pages are
// split into parts of up to C steps, a workgroup each, a sequence's own into parts of
// up to C over the wavefronts of a workgroup, a wavefront each. The last part of a
// unit is not full, by one half on average and by more in a unit shorter than C: C is
// all units' steps over the workgroups wanted less those, so that what runs at once is
// filled and no few parts are left to run after it (four groups of 80 rows: 303 ->
// 284 us). Parts are numbered group by group, then sequence by sequence. There are at
// most total / C, so at most `target`, workgroups plus one part per (unit, row block,
// head): the grid. The sums are float32, their rounding well inside the slack taken of
// C: every wavefront of the launch finds the same C, from the same operations.
__device__ __forceinline__ int steps_of(const Unit &u) { return (u.pages + 1) / 2; }
__device__ __forceinline__ int blocks_of(const SharedArgs &a, const Unit &u, bool shared) {
  const int br = shared ? kRows : a.own_rows;
  return div_small(u.rows + br - 1, br);
}
__device__ __forceinline__ Unit unit_of(const SharedArgs &a, bool shared, int i) {
  if (i >= (shared ? a.num_groups : a.batch)) return Unit{0, 0, 0, 0};
  return shared ? group_unit(a, i) : seq_unit(a, i);
}
__device__ __forceinline__ int parts_of(const Unit &u, int len) {
  return div_small(steps_of(u) + len - 1, len);
}

// Steps of a part of a group's pages, and of a sequence's own. sum(f): that of
// f(steps, row blocks, whether it is a group) of all units.
struct Lengths {
  int of[2];
};
template <int WAVES, class Sum>
__device__ __forceinline__ Lengths part_lengths(const SharedArgs &a, Sum sum) {
  const float total = sum([](float steps, float blocks, bool) { return steps * blocks; }) * a.Hkv;
  const float per = (float)a.target / fmaxf(total, 1.f);
  const float unfilled = sum([&](float steps, float blocks, bool shared) {
    const float full = steps * per * (shared ? 1.f : (float)WAVES);   // parts, were they all full
    return fmaxf(0.5f, 1.f - full) * blocks * (shared ? 1.f : 1.f / WAVES);
  }) * a.Hkv;
  const float wanted = fmaxf((float)a.target - unfilled, 0.5f * a.target);
  const float most = fmaxf(total * 1.0001f / wanted, (float)a.least);
  return Lengths{{(int)fminf(ceilf(most), 1e9f),
                  max((int)fminf(ceilf(most / WAVES), 1e9f), a.own_least)}};
}
template <class F>
__device__ __forceinline__ float of_unit(const SharedArgs &a, const Unit &u, bool shared, F f) {
  return f((float)steps_of(u), (float)(u.pages > 0 ? blocks_of(a, u, shared) : 0), shared);
}

// Part `off` of the n_split * row blocks * KV heads of a unit whose first is part e.
__device__ __forceinline__ void set_part(const SharedArgs &a, Item &it, bool shared, int unit, int e,
                                         int off) {
  it.shared = shared;
  it.unit = unit;
  it.row0 = (shared ? 0 : a.own_base) + (int64_t)e * (shared ? kRows : a.own_rows);
  const int block = div_small(off, it.n_split);
  it.split = off - block * it.n_split;
  it.rb = div_small(block, a.Hkv);
  it.g = block - it.rb * a.Hkv;
}

// The map of a large batch is made once, by a workgroup before the others start:
// a.map holds the part lengths, the workgroups of shared parts, the parts of
// sequences, then the first part of every group and of every sequence.
constexpr int kPlanThreads = 1024, kMapHead = 4;

template <int WAVES>
__global__ __launch_bounds__(kPlanThreads) void shared_plan_kernel(SharedArgs a) {
  __shared__ float s_sum[kPlanThreads / 64];
  __shared__ int s_run[kPlanThreads / 64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  auto sum = [&](auto f) {
    float x = 0.f;
    for (int i = threadIdx.x; i < a.num_groups; i += kPlanThreads)
      x += of_unit(a, unit_of(a, true, i), true, f);
    for (int i = threadIdx.x; i < a.batch; i += kPlanThreads)
      x += of_unit(a, unit_of(a, false, i), false, f);
    x = wave_sum(x);
    __syncthreads();
    if (lane == 0) s_sum[wave] = x;
    __syncthreads();
    x = 0.f;
    for (int w = 0; w < kPlanThreads / 64; ++w) x += s_sum[w];
    return x;
  };
  const Lengths len = part_lengths<WAVES>(a, sum);
  int32_t *first = a.map + kMapHead;
  for (int kind = 0; kind < 2; ++kind) {
    const bool shared = kind == 0;
    const int n = shared ? a.num_groups : a.batch;
    int base = 0;
    for (int i0 = 0; i0 < n; i0 += kPlanThreads) {
      const int i = i0 + threadIdx.x;
      const Unit u = unit_of(a, shared, i);
      const int cnt = parts_of(u, len.of[kind]) * blocks_of(a, u, shared) * a.Hkv;
      const int incl = wave_scan_add(cnt);
      __syncthreads();
      if (lane == 63) s_run[wave] = incl;
      __syncthreads();
      int before = base;
      for (int w = 0; w < kPlanThreads / 64; ++w) {
        if (w < wave) before += s_run[w];
        base += s_run[w];
      }
      if (i < n) first[i] = before + incl - cnt;
    }
    if (threadIdx.x == 0) {
      a.map[kind] = len.of[kind];
      a.map[2 + kind] = base;
    }
    first += n;
  }
}

template <int WAVES>
__device__ bool planned_item(const SharedArgs &a, int w, int wave, Item &it) {
  const int lane = threadIdx.x & 63;
  const bool shared = w < a.map[2];
  const int32_t *first = a.map + kMapHead + (shared ? 0 : a.num_groups);
  if (!shared) {
    w = (w - a.map[2]) * WAVES + wave;
    if (w >= a.map[3]) return false;
  }
  // the last unit whose first part is w or before
  int lo = 0, hi = shared ? a.num_groups : a.batch;
  while (hi - lo > 1) {
    const int step = (hi - lo + 63) / 64, i = lo + lane * step;
    const unsigned long long m = __ballot(i < hi && first[min(i, hi - 1)] <= w);
    lo += (__popcll(m) - 1) * step;
    hi = min(lo + step, hi);
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  const Unit u = unit_of(a, shared, lo);
  it.seq0 = __builtin_amdgcn_readfirstlane(u.seq0);
  it.rows = __builtin_amdgcn_readfirstlane(u.rows);
  it.page0 = __builtin_amdgcn_readfirstlane(u.page0);
  it.pages = __builtin_amdgcn_readfirstlane(u.pages);
  it.n_split = __builtin_amdgcn_readfirstlane(parts_of(u, a.map[shared ? 0 : 1]));
  const int e = __builtin_amdgcn_readfirstlane(first[lo]);
  if (it.n_split < 1) return false;            // (offsets that do not ascend)
  set_part(a, it, shared, lo, e, w - e);
  return true;
}

template <int WAVES>
__device__ bool shared_map(const SharedArgs &a, int w, int wave, Item &it) {
  if (a.map) return planned_item<WAVES>(a, w, wave, it);
  const int lane = threadIdx.x & 63;
  Unit first[2];                               // of the first 64, kept for the later passes
  first[0] = unit_of(a, true, lane);
  first[1] = unit_of(a, false, lane);
  const Lengths len = part_lengths<WAVES>(a, [&](auto f) {
    float x = of_unit(a, first[0], true, f) + of_unit(a, first[1], false, f);
    for (int i0 = 64; i0 < a.num_groups; i0 += 64) x += of_unit(a, unit_of(a, true, i0 + lane), true, f);
    for (int i0 = 64; i0 < a.batch; i0 += 64) x += of_unit(a, unit_of(a, false, i0 + lane), false, f);
    return wave_sum(x);
  });
  int base = 0;
  for (int kind = 0; kind < 2; ++kind) {
    const bool shared = kind == 0;
    const int n = shared ? a.num_groups : a.batch;
    if (!shared) {                             // parts are wavefronts' from here on
      w = (w - base) * WAVES + wave;
      base = 0;
    }
    for (int i0 = 0; i0 < n; i0 += 64) {
      const Unit u = i0 == 0 ? first[kind] : unit_of(a, shared, i0 + lane);
      const int parts = parts_of(u, len.of[kind]);
      const int cnt = parts * blocks_of(a, u, shared) * a.Hkv;
      const int incl = wave_scan_add(cnt), excl = incl - cnt;
      const unsigned long long hit = __ballot(w >= base + excl && w < base + incl);
      if (hit) {
        const int l = __builtin_amdgcn_readfirstlane(__ffsll((long long)hit) - 1);
        it.seq0 = __builtin_amdgcn_readlane(u.seq0, l);
        it.rows = __builtin_amdgcn_readlane(u.rows, l);
        it.page0 = __builtin_amdgcn_readlane(u.page0, l);
        it.pages = __builtin_amdgcn_readlane(u.pages, l);
        it.n_split = __builtin_amdgcn_readlane(parts, l);
        const int e = base + __builtin_amdgcn_readlane(excl, l);
        set_part(a, it, shared, i0 + l, e, w - e);
        return true;
      }
      base += lane63(incl);
    }
  }
  return false;
}

// ---------------------------------------------------------------------------
// operands
// ---------------------------------------------------------------------------

// An operand as loaded (fp8: codes, widened at use). A K operand serves 16 dims
// (float32: 8) of a step's 32 keys, a V operand 32 dims of a page's 16 keys
// (float32: of eight of them).
template <int KV> struct Operand { u32x4 x; };
template <> struct Operand<kFP8> { u32x2 x; };

// K operands of a step, as many as V operands; V operands per 32 dims.
template <int KV, int D> constexpr int operands() { return KV == kF32 ? D / 8 : D / 16; }
template <int KV> constexpr int v_parts() { return KV == kF32 ? 4 : 2; }

// Q^T, the operand K meets: 16-bit dims 16 c + 8 hb .., float32 8 c + 4 hb .. In
// registers, except 256-dim float32 heads' (128 of them): in LDS, lane for lane.
template <int KV, int D> constexpr bool q_in_lds() { return KV == kF32 && D == 256; }
template <int KV, int D> struct Queries {
  u32x4 q[q_in_lds<KV, D>() ? 1 : operands<KV, D>()];
  const u32x4 *lds;
  __device__ u32x4 at(int c) const {
    if constexpr (q_in_lds<KV, D>()) return lds[c * 64];
    else return q[c];
  }
};

__device__ __forceinline__ u32x4 widen8(u32x2 x) {
  const u32x2 lo = fp8x4_to_bf16x4(x[0]), hi = fp8x4_to_bf16x4(x[1]);
  return u32x4{lo[0], lo[1], hi[0], hi[1]};
}
__device__ __forceinline__ u32x4 wide(const Operand<kBF16> &r) { return r.x; }
__device__ __forceinline__ u32x4 wide(const Operand<kF32> &r) { return r.x; }
__device__ __forceinline__ u32x4 wide(const Operand<kFP8> &r) { return widen8(r.x); }

// The two pages of a step: ids (0 where there is none) and whether they are there.
struct Step {
  int id[2];
  bool ok[2];
};

// Operands of a step in memory, for the lane that multiplies them.
template <int KV, int D>
struct Pages {
  static constexpr size_t kTile = (size_t)kPage * D * elem_bytes(KV);
  const char *k, *v[2];
  // not live: the loads are issued all the same, all lanes' from one place (a branch
  // around them would leave the compiler no count of what is in flight, and make
  // every wait one for everything)
  __device__ Pages(const SharedArgs &a, const int (&id)[2], int g, int lane, bool live = true) {
    const int i = lane & 31, hb = lane >> 5, tok = key_of_row<KV>(i) & 15;
    const int k_at = tok * 8 * elem_bytes(KV) + hb * (KV == kF32 ? 16 : 128 * elem_bytes(KV));
    const int v_at = i * 16 * elem_bytes(KV) + hb * (KV == kF32 ? 16 : 8 * elem_bytes(KV));
    k = static_cast<const char *>(a.k_pages) +
        ((size_t)(i < 16 && live ? id[0] : id[1]) * a.Hkv + g) * kTile + (live ? k_at : 0);
#pragma unroll
    for (int pg = 0; pg < 2; ++pg)
      v[pg] = static_cast<const char *>(a.v_pages) + ((size_t)id[pg] * a.Hkv + g) * kTile +
              (live ? v_at : 0);
  }
  __device__ Operand<KV> raw_key(int c) const {
    return *reinterpret_cast<const Operand<KV> *>(k + c * (KV == kF32 ? 512 : 256 * elem_bytes(KV)));
  }
  __device__ Operand<KV> raw_value(int y, int db) const {
    if constexpr (KV == kF32)
      return *reinterpret_cast<const Operand<KV> *>((y >> 1 ? v[1] : v[0]) + db * 2048 + (y & 1) * 32);
    else
      return *reinterpret_cast<const Operand<KV> *>((y ? v[1] : v[0]) + db * 512 * elem_bytes(KV));
  }
  __device__ u32x4 key(int c) const { return wide(raw_key(c)); }
  __device__ u32x4 value(int y, int db) const { return wide(raw_value(y, db)); }
};

// The same in registers.
template <int KV, int D>
struct Held {
  Operand<KV> k[operands<KV, D>()], v[v_parts<KV>()][D / 32];
  __device__ __forceinline__ void load_k(const Pages<KV, D> &p) {
#pragma unroll
    for (int c = 0; c < operands<KV, D>(); ++c) k[c] = p.raw_key(c);
  }
  __device__ __forceinline__ void load_v(const Pages<KV, D> &p) {
#pragma unroll
    for (int y = 0; y < v_parts<KV>(); ++y)
#pragma unroll
      for (int db = 0; db < D / 32; ++db) v[y][db] = p.raw_value(y, db);
  }
  __device__ u32x4 key(int c) const { return wide(k[c]); }
  __device__ u32x4 value(int y, int db) const { return wide(v[y][db]); }
};

template <int KV, int D, class Source>
__device__ __forceinline__ f32x16 logits(const Source &src, const Queries<KV, D> &q) {
  // operands whose loads the compiler may have in flight together
  constexpr int kTogether = 8, K = operands<KV, D>();
  f32x16 s = zero16();
#pragma unroll
  for (int c0 = 0; c0 < K; c0 += kTogether) {
    u32x4 k[kTogether];
#pragma unroll
    for (int c = 0; c < kTogether; ++c)
      if (c0 + c < K) k[c] = src.key(c0 + c);
#pragma unroll
    for (int c = 0; c < kTogether; ++c) {
      if (c0 + c >= K) continue;
      const u32x4 qq = q.at(c0 + c);
      if constexpr (KV == kF32) {
#pragma unroll
        for (int e = 0; e < 4; ++e) s = mfma(__uint_as_float(k[c][e]), __uint_as_float(qq[e]), s);
      } else {
        s = mfma(k[c], qq, s);
      }
    }
    if (K > kTogether) __builtin_amdgcn_sched_barrier(0);
  }
  return s;
}

// ---------------------------------------------------------------------------
// one wavefront's share: 32 rows over its steps
// ---------------------------------------------------------------------------

template <int D> struct State {
  f32x16 o[D / 32];  // O^T: dims 32 db + (r % 4) + 8 (r / 4) + 4 hb of row lane % 32
  float ref, sum;    // reference (powers of two), and this lane's half of the sum
};

// Moves the reference above a step's logits (c z: in powers of two, c >= 0). MASKED: what
// weighs nothing against it goes, infinities and NaN too.
template <int D, bool MASKED>
__device__ __forceinline__ void move_reference(State<D> &st, const f32x16 &z, float c) {
  float top = max_f(z[0], z[1]);
#pragma unroll
  for (int i = 2; i < 16; ++i) top = max_f(top, z[i]);
  top *= c;
  if (__any(top > st.ref)) {
    top = max_f(top, other_half(top));
    const float ref = top > st.ref ? top + kDefer : st.ref;
    const float f = exp2_fast(st.ref - ref);
    st.ref = ref;
    st.sum *= f;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i)
        st.o[db][i] = MASKED && f == 0.f ? 0.f : st.o[db][i] * f;
  }
}
// Weights in the place of the logits.
template <int D>
__device__ __forceinline__ void weigh(State<D> &st, f32x16 &z, float c) {
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    z[i] = exp2_fast(fmaf(z[i], c, -st.ref));
    st.sum += z[i];
  }
}

// bf16 parts of a page's eight weights of a lane.
__device__ __forceinline__ void split8(const float *w, u32x4 &hi, u32x4 &lo, u32x4 &rest) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float x = w[2 * i], y = w[2 * i + 1];
    hi[i] = round_bf16x2(x, y);
    const float dx = less_bf16<false>(hi[i], x), dy = less_bf16<true>(hi[i], y);
    lo[i] = round_bf16x2(dx, dy);
    rest[i] = round_bf16x2(less_bf16<false>(lo[i], dx), less_bf16<true>(lo[i], dy));
  }
}

// What of a V operand's words (two bf16 values, or one float32) some row sees,
// from `seen` (bit r: key_of_reg(r) of this half of the wavefront is).
template <int KV>
__device__ __forceinline__ u32x4 seen_words(uint32_t seen, int y) {
  u32x4 m;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (KV == kF32)
      m[i] = (uint32_t)__builtin_amdgcn_sbfe((int)seen, 4 * y + i, 1);
    else
      m[i] = ((uint32_t)__builtin_amdgcn_sbfe((int)seen, 8 * y + 2 * i, 1) & 0xffffu) |
             ((uint32_t)__builtin_amdgcn_sbfe((int)seen, 8 * y + 2 * i + 1, 1) & 0xffff0000u);
  }
  return m;
}
// All ones where a value of the words is infinite or NaN.
template <int KV>
__device__ __forceinline__ u32x4 wild_words(u32x4 v) {
  u32x4 m;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (KV == kF32) {
      m[i] = (uint32_t)((int)((v[i] & 0x7f800000u) + 0x00800000u) >> 31);
    } else {
      const uint32_t b = ((v[i] & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
      m[i] = (b - (b >> 15)) | b;
    }
  }
  return m;
}
// 1 where a value of the words is +inf (class 0), -inf (1) or NaN (2).
template <int KV>
__device__ __forceinline__ u32x4 class_words(u32x4 v, int cls) {
  u32x4 m;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (KV == kF32) {
      const bool is = cls == 2 ? (v[i] & 0x7fffffffu) > 0x7f800000u
                               : v[i] == (cls == 0 ? 0x7f800000u : 0xff800000u);
      m[i] = is ? 0x3f800000u : 0u;
    } else {
      auto is = [&](uint32_t h) {
        return cls == 2 ? (h & 0x7fffu) > 0x7f80u : h == (cls == 0 ? 0x7f80u : 0xff80u);
      };
      m[i] = (is(v[i] & 0xffffu) ? 0x3f80u : 0u) | (is(v[i] >> 16) ? 0x3f800000u : 0u);
    }
  }
  return m;
}

// Infinities and NaNs of V that were kept out of the products: added by class to
// the rows that give them a weight.
template <int KV, int D, class Source>
__device__ __forceinline__ void add_classes(State<D> &st, const Source &src, const f32x16 &w,
                                            uint32_t seen) {
  for (int cls = 0; cls < 3; ++cls) {
    const float what = cls == 0 ? INFINITY : (cls == 1 ? -INFINITY : __builtin_nanf(""));
#pragma unroll
    for (int db = 0; db < D / 32; ++db) {
      f32x16 hits = zero16();
#pragma unroll
      for (int y = 0; y < v_parts<KV>(); ++y) {
        const u32x4 one = class_words<KV>(src.value(y, db) & seen_words<KV>(seen, y), cls);
        if constexpr (KV == kF32) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            hits = mfma(__uint_as_float(one[e]), w[4 * y + e] != 0.f ? 1.f : 0.f, hits);
        } else {
          u32x4 nz;
#pragma unroll
          for (int i = 0; i < 4; ++i)
            nz[i] = (w[8 * y + 2 * i] != 0.f ? 0x3f80u : 0u) |
                    (w[8 * y + 2 * i + 1] != 0.f ? 0x3f800000u : 0u);
          hits = mfma(one, nz, hits);
        }
      }
#pragma unroll
      for (int i = 0; i < 16; ++i)
        st.o[db][i] += hits[i] != 0.f ? what : 0.f;
      __builtin_amdgcn_sched_barrier(0);
    }
  }
}

// O += V^T P^T for a step's weights w. MASKED: some key of the step is hidden
// from some row. V of keys that no row sees is cleared, and infinities and NaNs
// of the others are kept out of the products, where a weight of zero would spread
// them, and added by class where the weight is not zero.
template <int KV, int D, bool MASKED, class Source>
__device__ __forceinline__ void add_values(State<D> &st, const Source &src, const f32x16 &w,
                                           uint32_t seen, const float (&vs)[2]) {
  uint32_t wild = 0;
#pragma unroll
  for (int y = 0; y < v_parts<KV>(); ++y) {
    u32x4 hi, lo, rest, sees;
    if constexpr (KV != kF32) {
      float p[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        // (MASKED: of a page that is not there or that a row does not see, the scale may
        // be anything)
        if constexpr (KV != kFP8) p[i] = w[8 * y + i];
        else if constexpr (MASKED) p[i] = w[8 * y + i] == 0.f ? 0.f : w[8 * y + i] * vs[y];
        else p[i] = w[8 * y + i] * vs[y];
      }
      split8(p, hi, lo, rest);
    }
    if constexpr (MASKED) sees = seen_words<KV>(seen, y);
#pragma unroll
    for (int db = 0; db < D / 32; ++db) {
      u32x4 v = src.value(y, db);
      if constexpr (MASKED) {
        v &= sees;
        const u32x4 m = wild_words<KV>(v);
        wild |= m[0] | m[1] | m[2] | m[3];
        v &= ~m;
      }
      if constexpr (KV == kF32) {
#pragma unroll
        for (int e = 0; e < 4; ++e) st.o[db] = mfma(__uint_as_float(v[e]), w[4 * y + e], st.o[db]);
      } else {
        st.o[db] = mfma(v, hi, st.o[db]);
        st.o[db] = mfma(v, lo, st.o[db]);
        st.o[db] = mfma(v, rest, st.o[db]);
      }
    }
    if (MASKED || KV == kF32) __builtin_amdgcn_sched_barrier(0);
  }
  if constexpr (MASKED)
    if (__any(wild != 0u)) add_classes<KV, D>(st, src, w, seen);
}

// The rows of a block that a lane serves.
struct RowOf {
  int64_t q;         // row in q (and out); -1: none
  int limit;         // keys it sees
};
__device__ __forceinline__ RowOf row_of(const SharedArgs &a, const Item &it, int r) {
  if (r >= it.rows) return RowOf{-1, 0};
  const int per = a.q_len * a.G;
  const int b = it.seq0 + r / per, rr = r % per, i = rr / a.G;
  // (2^27 pages hold one position more than 32 bits count: less one here)
  const int most = (int)min((long long)a.max_pages * kPage, 0x7fffffffll);
  return RowOf{((int64_t)b * a.q_len + i) * a.Hq + it.g * a.G + (rr - i * a.G),
               max(0, clamp_to(a.seq_lens[b], 0, most) - a.q_len + i + 1)};
}

// What a wavefront (or workgroup) walks: steps of table row `table`, whose first
// page is page `page0` of the sequence.
struct Walk {
  const int32_t *table;
  int page0, pages;
  int all, some;     // keys that every row, that some row sees
  int s0, s1;        // steps
  int plain;         // steps below this are there and seen by every row
};

__device__ __forceinline__ bool in_pool(const SharedArgs &a, int id) {
  return id >= 0 && (int64_t)id < a.num_pages;
}
// Page ids of a wavefront's steps first, first + stride, ..: 32 steps' in the lanes
// of one register, the next 32 steps' on the way. (A load of an id right before
// it is needed would be waited for with everything that is in flight.)
struct PageIds {
  int cur, next, k0, first, stride, lane;
  __device__ int fetch(const Walk &w, int k) const {
    const int e = 2 * (first + (k + (lane >> 1)) * stride) + (lane & 1);
    return w.table[min(e, max(w.pages - 1, 0))];
  }
  __device__ PageIds(const Walk &w, int first_, int stride_, int lane_)
      : k0(0), first(first_), stride(stride_), lane(lane_) {
    cur = fetch(w, 0);
    next = fetch(w, 32);
  }
  // of the k-th step; k never goes back
  __device__ Step at(const SharedArgs &a, const Walk &w, int k) {
    if (k - k0 >= 32) {
      k0 += 32;
      cur = next;
      next = fetch(w, k0 + 32);
    }
    const int s = first + k * stride;
    Step x;
#pragma unroll
    for (int pg = 0; pg < 2; ++pg) {
      const int id = __builtin_amdgcn_readlane(cur, 2 * (k - k0) + pg);
      x.ok[pg] = s < w.s1 && 2 * s + pg < w.pages && in_pool(a, id);
      x.id[pg] = x.ok[pg] ? id : 0;
    }
    return x;
  }
};
// What positions allow, if the pages of the wavefront's steps up to there are in the
// pool.
__device__ __forceinline__ int plain_steps(const SharedArgs &a, const Walk &w, const PageIds &ids) {
  const int end = max(w.s0, min(min(w.s1, w.pages / 2), (w.all / kPage - w.page0) / 2));
  bool fine = true;
  for (int k = 0; ids.first + k * ids.stride < end; k += 32) {
    const int id = k == 0 ? ids.cur : (k == 32 ? ids.next : ids.fetch(w, k));
    const int s = ids.first + (k + (ids.lane >> 1)) * ids.stride;
    fine &= s >= end || in_pool(a, id);
  }
  return __any(!fine) ? w.s0 : end;
}

// Raw logits to powers of two, up to the factor that is returned (not negative:
// the sign of sm_scale is in Q). MASKED: keys that a row does not see to -inf.
template <int KV, bool MASKED>
__device__ __forceinline__ float scale_logits(const SharedArgs &a, const Walk &w, f32x16 &z,
                                              uint32_t &seen, int s, const bool (&ok)[2], int limit,
                                              const float (&ks)[2], int lane) {
  const int hb = lane >> 5;
  seen = 0xffffu;
  if constexpr (KV != kFP8 && !MASKED) return a.scale_log2;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    z[i] *= KV == kFP8 ? a.scale_log2 * ks[i >> 3] : a.scale_log2;
    if constexpr (MASKED) {
      const int pos = (w.page0 + 2 * s + (i >> 3)) * kPage + key_of_reg<KV>(i & 7, hb);
      if (!(ok[i >> 3] && pos < limit)) z[i] = -INFINITY;
      if (!(ok[i >> 3] && pos < w.some)) seen &= ~(1u << i);
    }
  }
  return 1.f;
}

// One step with its operands; ks, vs: the pages' scales (fp8).
template <int KV, int D, bool MASKED, class Source>
__device__ __forceinline__ void take_step(State<D> &st, const SharedArgs &a, const Walk &w,
                                          const Queries<KV, D> &q, const Source &src, int s,
                                          const bool (&ok)[2], int limit, const float (&ks)[2],
                                          const float (&vs)[2], int lane) {
  f32x16 z = logits<KV, D>(src, q);
  uint32_t seen;
  const float c = scale_logits<KV, MASKED>(a, w, z, seen, s, ok, limit, ks, lane);
  move_reference<D, MASKED>(st, z, c);
  weigh(st, z, c);
  add_values<KV, D, MASKED>(st, src, z, seen, vs);
}

template <int KV>
__device__ __forceinline__ void scales_of(const SharedArgs &a, const int (&id)[2], float (&ks)[2],
                                          float (&vs)[2]) {
  if constexpr (KV == kFP8) {
#pragma unroll
    for (int pg = 0; pg < 2; ++pg) {
      ks[pg] = a.kv_scales[2 * (size_t)id[pg]];
      vs[pg] = a.kv_scales[2 * (size_t)id[pg] + 1];
    }
  }
}

// Whether steps that every row sees in full have a loop of their own, without masks.
template <int KV, int D> constexpr bool has_plain() { return KV != kF32 || D < 256; }

// Steps first, first + stride, .. below w.s1, operands from memory.
template <int KV, int D>
__device__ __forceinline__ void walk_memory(State<D> &st, const SharedArgs &a, const Walk &w,
                                            const Queries<KV, D> &q, int g, PageIds ids, int limit) {
  const int lane = ids.lane, first = ids.first, stride = ids.stride;
  if (first >= w.s1) return;
  int k = 0;
  auto step = [&](int i) { return first + i * stride; };
  if constexpr (has_plain<KV, D>()) {
    // the next step's K is fetched as soon as this one's has been multiplied, and
    // so is V
    if (first < w.plain) {
      const bool fine[2] = {true, true};
      float ks[2] = {1.f, 1.f}, vs[2] = {1.f, 1.f}, ks1[2] = {1.f, 1.f}, vs1[2] = {1.f, 1.f};
      Held<KV, D> r;
      {
        const Step x = ids.at(a, w, 0);
        const Pages<KV, D> p(a, x.id, g, lane);
        r.load_k(p);
        r.load_v(p);
        scales_of<KV>(a, x.id, ks, vs);
      }
      for (;;) {
        const bool more = step(k + 1) < w.plain;
        const Step x = ids.at(a, w, k + 1);
        const Pages<KV, D> p(a, x.id, g, lane, more);
        scales_of<KV>(a, x.id, ks1, vs1);
        f32x16 z = logits<KV, D>(r, q);
        __builtin_amdgcn_sched_barrier(0);
        r.load_k(p);
        __builtin_amdgcn_sched_barrier(0);
        uint32_t seen;
        const float c = scale_logits<KV, false>(a, w, z, seen, step(k), fine, limit, ks, lane);
        move_reference<D, false>(st, z, c);
        weigh(st, z, c);
        add_values<KV, D, false>(st, r, z, seen, vs);
        __builtin_amdgcn_sched_barrier(0);
        r.load_v(p);
        ++k;
        if (!more) break;
#pragma unroll
        for (int pg = 0; pg < 2; ++pg) {
          ks[pg] = ks1[pg];
          vs[pg] = vs1[pg];
        }
      }
    }
  }
  for (; step(k) < w.s1; ++k) {
    const Step x = ids.at(a, w, k);
    float ks[2] = {1.f, 1.f}, vs[2] = {1.f, 1.f};
    scales_of<KV>(a, x.id, ks, vs);
    take_step<KV, D, true>(st, a, w, q, Pages<KV, D>(a, x.id, g, lane), step(k), x.ok, limit, ks, vs, lane);
  }
}

// ---------------------------------------------------------------------------
// the kernel
// ---------------------------------------------------------------------------

// A launch has fewer than 2^32 threads along x: workgroups from here on go to z.
constexpr long long kAlongX = 1ll << 21;
__device__ __forceinline__ unsigned flat_block() {
  return blockIdx.z * (unsigned)kAlongX + blockIdx.x;
}

template <int KV, int D>
struct Layout {
  static constexpr int kWaves = waves_of(KV, D);
  // the wavefronts' parts, 32 dims at a time: [wave][row][32 dims + 4]
  static constexpr int kPart = kRows * 36 * 4;
  static constexpr int kQ = kWaves * kPart;
  static constexpr int kBytes = kQ + (q_in_lds<KV, D>() ? kWaves * operands<KV, D>() * 1024 : 0);
};

template <int KV, int D>
__global__ __launch_bounds__(64 * waves_of(KV, D))
__attribute__((amdgpu_waves_per_eu(waves_of(KV, D) / 4)))
void attn_shared_kernel(SharedArgs a) {
  constexpr int kWaves = waves_of(KV, D);
  __shared__ __align__(16) char smem[Layout<KV, D>::kBytes];
  __shared__ float s_m[kWaves][kRows], s_l[kWaves][kRows];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int hb = lane >> 5;
  Item it;
  if (!shared_map<kWaves>(a, (int)flat_block(), wave, it)) return;   // (a shared part: all wavefronts)
  const int slot_rows = it.shared ? kRows : a.own_rows;
  const int64_t part0 =
      it.row0 + ((int64_t)(it.rb * a.Hkv + it.g) * it.n_split + it.split) * slot_rows;
  // (group offsets that do not ascend)
  if (part0 + slot_rows > (it.shared ? a.own_base : a.part_rows)) return;
  if (it.rb == 0 && it.g == 0 && it.split == 0 && (it.shared ? threadIdx.x == 0 : lane == 0))
    (it.shared ? a.group_parts : a.seq_parts)[it.unit] = PartsOf{it.row0, it.n_split, 0};

  // ---- steps, a workgroup's wavefronts in turn ------------------------------------
  Walk w;
  w.table = a.table + (size_t)it.seq0 * a.stride + it.page0;
  w.page0 = it.page0;
  w.pages = it.pages;
  const int steps = (it.pages + 1) / 2;
  w.s0 = (int)((long long)steps * it.split / it.n_split);
  w.s1 = (int)((long long)steps * (it.split + 1) / it.n_split);
  const int first = w.s0 + (it.shared ? wave : 0), stride = it.shared ? kWaves : 1;
  PageIds ids(w, first, stride, opaque(lane));

  // ---- rows ---------------------------------------------------------------------
  const int r0 = it.rb * slot_rows, rr = lane & 31;     // of the unit, of the block
  const RowOf row = row_of(a, it, rr < slot_rows ? r0 + rr : it.rows);
  Queries<KV, D> q;
  {
    constexpr int kBytes = KV == kF32 ? 4 : 2;
    const char *p = static_cast<const char *>(a.q) + (row.q < 0 ? 0 : row.q) * D * kBytes + hb * 16;
    u32x4 *lds = reinterpret_cast<u32x4 *>(smem + Layout<KV, D>::kQ) +
                 wave * operands<KV, D>() * 64 + lane;
    q.lds = lds;
#pragma unroll
    for (int c = 0; c < operands<KV, D>(); ++c) {
      u32x4 x = row.q < 0 ? u32x4{0, 0, 0, 0} : *reinterpret_cast<const u32x4 *>(p + c * 32);
      x ^= a.q_sign;
      if constexpr (q_in_lds<KV, D>()) lds[c * 64] = x;   // read by this lane alone
      else q.q[c] = x;
    }
  }
  // Rows that see nothing (a padded sequence's) are walked as if they saw everything,
  // and have no weight afterwards: the other rows' steps stay without masks.
  int all = row.limit == 0 ? 0x7fffffff : row.limit, some = row.limit;
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) {
    all = min(all, __shfl_xor(all, o, 64));
    some = max(some, __shfl_xor(some, o, 64));
  }
  w.all = __builtin_amdgcn_readfirstlane(all);
  w.some = __builtin_amdgcn_readfirstlane(some);
  // A product gives 0 * inf = NaN where a weight, or one of its parts, is zero, and
  // inf - inf where two parts differ in sign. Rather than test V on the way, a wavefront
  // whose result is not finite walks its steps again with masks, which keep infinities
  // and NaN of V out of the products. (Not for rows that see nothing, nor for those
  // that a NaN logit has made NaN.) The lane is opaque, or addresses and page ids would
  // be kept from walk to walk (15 registers more than 256-dim bf16 has). The test and
  // what it keeps cost 0.3 us of 26.7 (8 x 16K, bf16) and 3 of 291 (fp8 windows).
  State<D> st;
  w.plain = plain_steps(a, w, ids);
  for (;;) {
#pragma unroll
    for (int db = 0; db < D / 32; ++db) st.o[db] = zero16();
    st.ref = kNoMax;
    st.sum = 0.f;
    walk_memory<KV, D>(st, a, w, q, it.g, ids, row.limit);
    st.sum += other_half(st.sum);
    if (!has_plain<KV, D>() || w.plain <= first) break;
    float top = 0.f;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) top = max_f(top, __builtin_fabsf(st.o[db][i]));
    if (!__any(!(top < INFINITY) && row.limit > 0 && st.sum == st.sum)) break;
    w.plain = w.s0;
    ids = PageIds(w, first, stride, opaque(lane));
  }
  if (row.limit == 0) {
    st.sum = 0.f;
    st.ref = kNoMax;
  }
  if (!it.shared) {
    // ---- a wavefront by itself ----------------------------------------------------
    if (rr >= slot_rows || r0 + rr >= it.rows) return;
    const float inv = st.sum == 0.f ? 0.f : 1.f / st.sum;
    float *o = a.part_o + (part0 + rr) * D;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        f32x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = st.sum == 0.f ? 0.f : st.o[db][4 * y + e] * inv;
        *reinterpret_cast<f32x4 *>(o + 32 * db + 8 * y + 4 * hb) = v;
      }
    if (hb == 0) a.part_lse[part0 + rr] = st.sum == 0.f ? -INFINITY : st.ref + log2f(st.sum);
    return;
  }

  // ---- a workgroup: its wavefronts' parts, of the same rows ------------------------
  if (lane < kRows) {
    s_m[wave][lane] = st.ref;
    s_l[wave][lane] = st.sum;
  }
  __syncthreads();
  float *part = reinterpret_cast<float *>(smem);
  float m = s_m[0][rr];
#pragma unroll
  for (int t = 1; t < kWaves; ++t) m = max_f(m, s_m[t][rr]);
  const float f = exp2_fast(st.ref - m);
  for (int db = 0; db < D / 32; ++db) {
    if (db) __syncthreads();
#pragma unroll
    for (int d = 0; d < D / 32; ++d)           // (registers are not indexed)
      if (d == db) {
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          f32x4 v;
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = f == 0.f ? 0.f : st.o[d][4 * y + e] * f;
          *reinterpret_cast<f32x4 *>(part + (wave * kRows + rr) * 36 + 8 * y + 4 * hb) = v;
        }
      }
    __syncthreads();
    for (int i = threadIdx.x; i < kRows * 8; i += 64 * kWaves) {
      const int rl = i >> 3, d = (i & 7) * 4;
      if (rl >= slot_rows || r0 + rl >= it.rows) continue;
      float mm = s_m[0][rl];
#pragma unroll
      for (int t = 1; t < kWaves; ++t) mm = max_f(mm, s_m[t][rl]);
      float l = 0.f;
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int t = 0; t < kWaves; ++t) {
        l += s_l[t][rl] * exp2_fast(s_m[t][rl] - mm);
        const f32x4 x = *reinterpret_cast<const f32x4 *>(part + (t * kRows + rl) * 36 + d);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] += x[e];
      }
      const float inv = l == 0.f ? 0.f : 1.f / l;
      f32x4 res;
#pragma unroll
      for (int e = 0; e < 4; ++e) res[e] = l == 0.f ? 0.f : o[e] * inv;
      *reinterpret_cast<f32x4 *>(a.part_o + (part0 + rl) * D + 32 * db + d) = res;
      if (db == 0 && d == 0) a.part_lse[part0 + rl] = l == 0.f ? -INFINITY : mm + log2f(l);
    }
  }
}

// ---------------------------------------------------------------------------
// merge: rows of (sequence, KV head) over the parts of its group and its own
// ---------------------------------------------------------------------------

constexpr int kItems = 128, kShares = 8;       // (row, four dims) items; threads an item

template <int D>
__global__ __launch_bounds__(kItems * kShares) void merge_shared_kernel(SharedArgs a) {
  constexpr int D4 = D / 4, kBatch = 4;
  __shared__ f32x4 s_o[kShares][kItems];
  __shared__ float s_m[kShares][kItems], s_l[kShares][kItems];
  const unsigned unit = flat_block();
  if (unit >= (unsigned)a.batch * (unsigned)a.Hkv) return;
  const int g = unit % (unsigned)a.Hkv, b = unit / (unsigned)a.Hkv;
  const int grp = group_of(a, b);
  const Unit own = seq_unit(a, b);
  Unit pre{0, 0, 0, 0};
  if (grp >= 0) pre = group_unit(a, grp);
  const PartsOf po = own.pages > 0 ? a.seq_parts[b] : PartsOf{0, 0, 0};
  const PartsOf pp = pre.pages > 0 ? a.group_parts[grp] : PartsOf{0, 0, 0};
  const int per = a.q_len * a.G;
  const int item = threadIdx.x % kItems, share = threadIdx.x / kItems;
  const int i = min((int)blockIdx.y * kItems + item, per * D4 - 1);
  const int r = i / D4, d = i % D4 * 4;
  float m = kNoMax, l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  auto fold = [&](float lse, f32x4 v) {
    if (lse == -INFINITY) return;              // no key seen
    const float mm = max_f(m, lse);
    const float f = exp2_fast(m - mm), w = exp2_fast(lse - mm);
    m = mm;
    l = l * f + w;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = (f == 0.f ? 0.f : o[e] * f) + (w == 0.f ? 0.f : v[e] * w);
  };
  auto add = [&](int64_t row0, int n, int rows, int rr) {
    if (n <= 0) return;
    const int rb = rr / rows;
    const int64_t at0 = row0 + (int64_t)(rb * a.Hkv + g) * n * rows + (rr - rb * rows);
    // (only with group offsets that do not ascend)
    if (row0 < 0 || n > a.most_parts || rr < 0 || at0 + (int64_t)(n - 1) * rows >= a.part_rows) return;
    for (int s = share; s < n; s += kShares * kBatch) {
      float lse[kBatch];
      f32x4 v[kBatch];
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const int64_t at = at0 + (int64_t)min(s + kShares * j, n - 1) * rows;
        lse[j] = s + kShares * j < n ? a.part_lse[at] : -INFINITY;
        v[j] = *reinterpret_cast<const f32x4 *>(a.part_o + at * D + d);
      }
#pragma unroll
      for (int j = 0; j < kBatch; ++j) fold(lse[j], v[j]);
    }
  };
  add(pp.row0, pp.n, kRows, (b - pre.seq0) * per + r);
  add(po.row0, po.n, a.own_rows, r);
  s_o[share][item] = o;
  s_m[share][item] = m;
  s_l[share][item] = l;
  __syncthreads();
  if (share != 0 || (int)blockIdx.y * kItems + item >= per * D4) return;
#pragma unroll
  for (int t = 1; t < kShares; ++t) {
    const float lt = s_l[t][item];
    if (lt == 0.f) continue;                   // nothing there (a sum is 0 only then; NaN is not)
    const float mt = s_m[t][item], mm = max_f(m, mt);
    const float f = exp2_fast(m - mm), w = exp2_fast(mt - mm);
    const f32x4 v = s_o[t][item];
    m = mm;
    l = l * f + lt * w;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = (f == 0.f ? 0.f : o[e] * f) + (w == 0.f ? 0.f : v[e] * w);
  }
  const int qi = r / a.G;
  const int64_t row = ((int64_t)b * a.q_len + qi) * a.Hq + g * a.G + (r - qi * a.G);
  f32x4 res;
#pragma unroll
  for (int e = 0; e < 4; ++e) res[e] = l == 0.f ? 0.f : o[e] / l;
  *reinterpret_cast<f32x4 *>(a.out + row * D + d) = res;
  if (d == 0) a.lse[row] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
}

template <int KV, int D>
void launch_d(const SharedArgs &a, hipStream_t s) {
  constexpr int kWaves = waves_of(KV, D);
  auto along = [](long long n) { return (unsigned)std::min(n, kAlongX); };
  auto above = [](long long n) { return (unsigned)((n + kAlongX - 1) / kAlongX); };
  const dim3 grid(along(a.grid), 1, above(a.grid)), block(64 * kWaves);
  if (a.map) hipLaunchKernelGGL(shared_plan_kernel<kWaves>, dim3(1), dim3(kPlanThreads), 0, s, a);
  hipLaunchKernelGGL((attn_shared_kernel<KV, D>), grid, block, 0, s, a);
  const int items = a.q_len * a.G * (D / 4);
  const long long units = (long long)a.batch * a.Hkv;
  hipLaunchKernelGGL(merge_shared_kernel<D>,
                     dim3(along(units), (unsigned)((items + kItems - 1) / kItems), above(units)),
                     dim3(kItems * kShares), 0, s, a);
}

template <int KV>
void launch_kv(const SharedArgs &a, hipStream_t s) {
  if (a.D == 64) launch_d<KV, 64>(a, s);
  else if (a.D == 128) launch_d<KV, 128>(a, s);
  else launch_d<KV, 256>(a, s);
}

}  // namespace

int shared_waves(int kv_type, int D) { return waves_of(kv_type, D); }

hipError_t launch_attn_shared(const SharedArgs &a, hipStream_t s) {
  if (a.kv_type == kF32) launch_kv<kF32>(a, s);
  else if (a.kv_type == kBF16) launch_kv<kBF16>(a, s);
  else launch_kv<kFP8>(a, s);
  return hipGetLastError();
}

}  // namespace kap

// Verification and decode attention of sequences that share leading pages
// (groups of requests over one document): the shared pages are walked once with
// the query rows of all the group's sequences, then every sequence's own pages
// with its own rows, and the parts are merged by their log-sum-exp.
//
// A unit is (rows, pages): a group's rows over its shared pages, or a
// sequence's q_len * G rows over its own. A workgroup owns (unit, block of rows,
// KV head, split of the pages). A wavefront holds 32 rows and walks 32 keys (two
// pages) a step:
//   S^T[key][row] = K . Q^T       v_mfma_f32_32x32x16_bf16, or
//   O^T[dim][row] += V^T P^T      v_mfma_f32_32x32x2_f32 for float32 KV
// The accumulator of S^T gives lane l row l % 32 and 16 of the keys, the other
// lane of that row the rest; with the keys of K's operand in the order of
// key_of_row() those are eight neighbouring keys of either page, which is the
// layout P^T's operand needs: weights never leave their lane.
//
// Weights are float32, split into bf16 hi + lo for 16-bit V, both rounded to
// nearest (what is left out is at most 2^-18 of a weight; with hi truncated
// outputs were off by 4.4e-6 of their norm). The reference they are taken against
// stays above every logit: when one exceeds it, it moves kDefer beyond (in powers
// of two), so that it hardly ever moves and no weight exceeds 1.
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

constexpr int kWaves = 4;
constexpr int kRows = 32;                      // of a wavefront
constexpr int kKeys = 32;                      // of a step

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

__device__ __forceinline__ long long wave_sum(long long x) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) x += __shfl_xor(x, o, 64);
  return x;
}

// Work item of workgroup w. A unit's cost is its steps times its row blocks and
// heads; a unit is split into ceil(steps / C) parts, where C, the cost of all
// units over the workgroups wanted, is the most a workgroup gets. Parts are
// numbered group by group, then sequence by sequence, so at most `target` plus
// one per (unit, row block, head) of them exist: the grid.
__device__ bool shared_map(const SharedArgs &a, int w, Item &it) {
  const int lane = threadIdx.x & 63;
  auto steps_of = [](const Unit &u) { return (u.pages + 1) / 2; };
  auto blocks_of = [&](const Unit &u, bool shared) {
    const int br = shared ? a.shared_rows : a.own_rows;
    return (u.rows + br - 1) / br;
  };
  auto unit_of = [&](bool shared, int i) {
    const int n = shared ? a.num_groups : a.batch;
    if (i >= n) return Unit{0, 0, 0, 0};
    return shared ? group_unit(a, i) : seq_unit(a, i);
  };
  long long total = 0;
  for (int kind = 0; kind < 2; ++kind) {
    const int n = kind == 0 ? a.num_groups : a.batch;
    for (int i0 = 0; i0 < n; i0 += 64) {
      const Unit u = unit_of(kind == 0, i0 + lane);
      total += wave_sum((long long)steps_of(u) * blocks_of(u, kind == 0) *
                        (kind == 0 ? a.shared_cost : a.own_cost));
    }
  }
  total *= a.Hkv;
  const long long most = max((total + a.target - 1) / a.target, (long long)a.least);
  int base = 0;
  int64_t row = 0;
  for (int kind = 0; kind < 2; ++kind) {
    const bool shared = kind == 0;
    const int n = shared ? a.num_groups : a.batch;
    const int slot_rows = shared ? a.shared_rows : a.own_rows;
    for (int i0 = 0; i0 < n; i0 += 64) {
      const Unit u = unit_of(shared, i0 + lane);
      const int rb = blocks_of(u, shared);
      const int parts =
          (int)ceil((double)steps_of(u) * (shared ? a.shared_cost : a.own_cost) / (double)most);
      const int cnt = parts * rb * a.Hkv;
      const int incl = wave_scan_add(cnt), excl = incl - cnt;
      const unsigned long long hit = __ballot(w >= base + excl && w < base + incl);
      if (hit) {
        const int l = __builtin_amdgcn_readfirstlane(__ffsll((long long)hit) - 1);
        it.shared = shared;
        it.unit = i0 + l;
        it.seq0 = __builtin_amdgcn_readlane(u.seq0, l);
        it.rows = __builtin_amdgcn_readlane(u.rows, l);
        it.page0 = __builtin_amdgcn_readlane(u.page0, l);
        it.pages = __builtin_amdgcn_readlane(u.pages, l);
        it.n_split = __builtin_amdgcn_readlane(parts, l);
        const int e = __builtin_amdgcn_readlane(excl, l);
        it.row0 = row + (int64_t)e * slot_rows;
        const int off = w - base - e;
        const int block = off / it.n_split;
        it.split = off - block * it.n_split;
        it.rb = block / a.Hkv;
        it.g = block - it.rb * a.Hkv;
        return true;
      }
      const int all = lane63(incl);
      base += all;
      row += (int64_t)all * slot_rows;
    }
  }
  return false;
}

// ---------------------------------------------------------------------------
// operands
// ---------------------------------------------------------------------------

// K and V^T operands as loaded (fp8: codes, widened at use): a K operand serves
// 16 dims (float32: 8) of the step's 32 keys, a V operand 32 dims of a page's 16
// keys (float32: of eight of them).
template <int KV> struct KOperand { u32x4 x; };
template <> struct KOperand<kFP8> { u32x2 x; };
template <int KV> using VOperand = KOperand<KV>;

// Q^T, the operand K meets: 16-bit dims 16 c + 8 hb .., float32 8 c + 4 hb .. In
// registers, except where they are 128 of them: 256-dim float32 heads keep it in
// LDS, lane for lane.
template <int KV, int D> constexpr int q_operands() { return KV == kF32 ? D / 8 : D / 16; }
template <int KV, int D> constexpr bool q_in_lds() { return KV == kF32 && D == 256; }
template <int KV, int D> struct Queries {
  u32x4 q[q_in_lds<KV, D>() ? 1 : q_operands<KV, D>()];
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
__device__ __forceinline__ u32x4 wide(const KOperand<kBF16> &r) { return r.x; }
__device__ __forceinline__ u32x4 wide(const KOperand<kF32> &r) { return r.x; }
__device__ __forceinline__ u32x4 wide(const KOperand<kFP8> &r) { return widen8(r.x); }

// The two pages of a step: ids (0 where there is none) and what is visible.
struct Step {
  int id[2];
  bool ok[2];
  int pos;           // of its first key
};

// Operands of a step from memory, in the lane that multiplies them.
template <int KV, int D>
struct Pages {
  static constexpr int kK = KV == kF32 ? D / 8 : D / 16;   // K operands
  static constexpr int kV = KV == kF32 ? 4 : 2;            // V operands per 32 dims
  const char *k, *v[2];
  __device__ Pages(const SharedArgs &a, const Step &s, int g, int lane) {
    constexpr size_t kTile = (size_t)kPage * D * elem_bytes(KV);
    const int i = lane & 31, hb = lane >> 5, tok = key_of_row<KV>(i) & 15;
    k = static_cast<const char *>(a.k_pages) +
        ((size_t)(i < 16 ? s.id[0] : s.id[1]) * a.Hkv + g) * kTile +
        tok * 8 * elem_bytes(KV) + hb * (KV == kF32 ? 16 : 128 * elem_bytes(KV));
#pragma unroll
    for (int pg = 0; pg < 2; ++pg)
      v[pg] = static_cast<const char *>(a.v_pages) + ((size_t)s.id[pg] * a.Hkv + g) * kTile +
              i * 16 * elem_bytes(KV) + hb * (KV == kF32 ? 16 : 8 * elem_bytes(KV));
  }
  __device__ KOperand<KV> key(int c) const {
    return *reinterpret_cast<const KOperand<KV> *>(k + c * (KV == kF32 ? 512 : 256 * elem_bytes(KV)));
  }
  __device__ VOperand<KV> value(int y, int db) const {
    if constexpr (KV == kF32)
      return *reinterpret_cast<const VOperand<KV> *>(v[y >> 1] + db * 2048 + (y & 1) * 32);
    else
      return *reinterpret_cast<const VOperand<KV> *>(v[y] + db * 512 * elem_bytes(KV));
  }
};

template <int KV, int D, class Source>
__device__ __forceinline__ f32x16 logits(const Source &src, const Queries<KV, D> &q) {
  // operands whose loads the compiler may have in flight together (more spill
  // with 256-dim float32 heads)
  constexpr int kTogether = KV == kF32 ? 8 : 16;
  f32x16 s = zero16();
#pragma unroll
  for (int c0 = 0; c0 < Source::kK; c0 += kTogether) {
    KOperand<KV> k[kTogether];
#pragma unroll
    for (int c = 0; c < kTogether; ++c)
      if (c0 + c < Source::kK) k[c] = src.key(c0 + c);
#pragma unroll
    for (int c = 0; c < kTogether; ++c) {
      if (c0 + c >= Source::kK) continue;
      const u32x4 kk = wide(k[c]), qq = q.at(c0 + c);
      if constexpr (KV == kF32) {
#pragma unroll
        for (int e = 0; e < 4; ++e) s = mfma(__uint_as_float(kk[e]), __uint_as_float(qq[e]), s);
      } else {
        s = mfma(kk, qq, s);
      }
    }
    if (Source::kK > kTogether) __builtin_amdgcn_sched_barrier(0);
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

// Weights of a step's logits (z: in powers of two), in place; moves the reference.
template <int D>
__device__ __forceinline__ void weigh(State<D> &st, f32x16 &z) {
  float top = max_f(z[0], z[1]);
#pragma unroll
  for (int i = 2; i < 16; ++i) top = max_f(top, z[i]);
  if (__any(top > st.ref)) {
    top = max_f(top, other_half(top));
    const float ref = top > st.ref ? top + kDefer : st.ref;
    const float f = exp2_fast(st.ref - ref);
    st.ref = ref;
    st.sum *= f;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) st.o[db][i] *= f;
  }
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    z[i] = exp2_fast(z[i] - st.ref);
    st.sum += z[i];
  }
}

// bf16 hi and lo parts of a page's eight weights of a lane.
__device__ __forceinline__ void split8(const float *w, u32x4 &hi, u32x4 &lo) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float x = w[2 * i], y = w[2 * i + 1];
    hi[i] = round_bf16x2(x, y);
    lo[i] = round_bf16x2(less_bf16<false>(hi[i], x), less_bf16<true>(hi[i], y));
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

// O += V^T P^T for a step's weights w. MASKED: some key of the step is hidden
// from some row. V of keys that no row sees is cleared, and infinities and NaNs
// of the others are kept out of the products, where a weight of zero would spread
// them, and added by class where the weight is not zero.
template <int KV, int D, bool MASKED, class Source>
__device__ __forceinline__ void add_values(State<D> &st, const Source &src, const f32x16 &w,
                                           uint32_t seen, const float (&vs)[2]) {
  uint32_t wild = 0;
#pragma unroll
  for (int y = 0; y < Source::kV; ++y) {
    u32x4 hi, lo, sees;
    if constexpr (KV != kF32) {
      float p[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) p[i] = KV == kFP8 ? w[8 * y + i] * vs[y] : w[8 * y + i];
      split8(p, hi, lo);
    }
    if constexpr (MASKED) sees = seen_words<KV>(seen, y);
    VOperand<KV> r[D / 32];
#pragma unroll
    for (int db = 0; db < D / 32; ++db) r[db] = src.value(y, db);
#pragma unroll
    for (int db = 0; db < D / 32; ++db) {
      u32x4 v = wide(r[db]);
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
      }
    }
    if (MASKED || Source::kV > 2) __builtin_amdgcn_sched_barrier(0);
  }
  if constexpr (MASKED) {
    if (!__any(wild != 0u)) return;
    for (int cls = 0; cls < 3; ++cls) {
      const float what = cls == 0 ? INFINITY : (cls == 1 ? -INFINITY : __builtin_nanf(""));
#pragma unroll
      for (int db = 0; db < D / 32; ++db) {
        f32x16 hits = zero16();
#pragma unroll
        for (int y = 0; y < Source::kV; ++y) {
          const u32x4 one = class_words<KV>(wide(src.value(y, db)) & seen_words<KV>(seen, y), cls);
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
  return RowOf{((int64_t)b * a.q_len + i) * a.Hq + it.g * a.G + (rr - i * a.G),
               max(0, min(a.seq_lens[b], a.max_pages * kPage) - a.q_len + i + 1)};
}

template <int KV, int D>
__global__ __launch_bounds__(64 * kWaves)
void attn_shared_kernel(SharedArgs a) {
  constexpr int DC = D < 128 ? D : 128;        // dims combined through LDS at a time
  __shared__ float s_o[kWaves][kRows][DC + 4];
  __shared__ float s_m[kWaves][kRows], s_l[kWaves][kRows];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int hb = lane >> 5;
  Item it;
  if (!shared_map(a, blockIdx.x, it)) return;
  const int slot_rows = it.shared ? a.shared_rows : a.own_rows;
  const int64_t part0 =
      it.row0 + ((int64_t)(it.rb * a.Hkv + it.g) * it.n_split + it.split) * slot_rows;
  if (part0 + slot_rows > a.part_rows) return;   // group offsets that do not ascend
  if (it.rb == 0 && it.g == 0 && it.split == 0 && threadIdx.x == 0)
    (it.shared ? a.group_parts : a.seq_parts)[it.unit] = PartsOf{it.row0, it.n_split, 0};

  const int r0 = it.rb * slot_rows;
  const RowOf row = row_of(a, it, (lane & 31) < slot_rows ? r0 + (lane & 31) : it.rows);
  Queries<KV, D> q;
  {
    constexpr int kBytes = KV == kF32 ? 4 : 2;
    const char *p = static_cast<const char *>(a.q) + (row.q < 0 ? 0 : row.q) * D * kBytes + hb * 16;
    __shared__ u32x4 s_q[q_in_lds<KV, D>() ? q_operands<KV, D>() * 64 : 1];
    q.lds = s_q + lane;
#pragma unroll
    for (int c = 0; c < q_operands<KV, D>(); ++c) {
      const u32x4 x = row.q < 0 ? u32x4{0, 0, 0, 0} : *reinterpret_cast<const u32x4 *>(p + c * 32);
      if constexpr (q_in_lds<KV, D>()) {
        if (wave == 0) s_q[c * 64 + lane] = x;
      } else {
        q.q[c] = x;
      }
    }
    if constexpr (q_in_lds<KV, D>()) __syncthreads();
  }
  // keys that every row, and that some row of the block sees
  int all = row.q < 0 ? 0x7fffffff : row.limit, some = row.limit;
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) {
    all = min(all, __shfl_xor(all, o, 64));
    some = max(some, __shfl_xor(some, o, 64));
  }
  all = __builtin_amdgcn_readfirstlane(all);
  some = __builtin_amdgcn_readfirstlane(some);

  const int steps = (it.pages + 1) / 2;
  const int s0 = (int)((long long)steps * it.split / it.n_split);
  const int s1 = (int)((long long)steps * (it.split + 1) / it.n_split);
  const int32_t *table = a.table + (size_t)it.seq0 * a.stride + it.page0;
  auto step_at = [&](int s) {
    Step x;
    x.pos = (it.page0 + 2 * s) * kPage;
#pragma unroll
    for (int pg = 0; pg < 2; ++pg) {
      const int id = 2 * s + pg < it.pages ? table[2 * s + pg] : -1;
      x.ok[pg] = id >= 0 && (int64_t)id < a.num_pages;
      x.id[pg] = x.ok[pg] ? id : 0;
    }
    return x;
  };

  State<D> st;
#pragma unroll
  for (int db = 0; db < D / 32; ++db) st.o[db] = zero16();
  st.ref = kNoMax;
  st.sum = 0.f;
  // Steps whose keys every row sees, then the rest: those at the end of a
  // sequence, and from the first page on that is not there.
  int s = s0 + wave;
  auto walk = [&](auto masked) {
    constexpr bool kMasked = decltype(masked)::value;
    for (; s < s1; s += kWaves) {
      const Step x = step_at(s);
      if (!kMasked && !(x.ok[0] && x.ok[1] && x.pos + kKeys <= all)) break;
      const Pages<KV, D> r(a, x, it.g, lane);
      float ks[2] = {1.f, 1.f}, vs[2] = {1.f, 1.f};
      if constexpr (KV == kFP8) {
#pragma unroll
        for (int pg = 0; pg < 2; ++pg) {
          ks[pg] = a.kv_scales[2 * (size_t)x.id[pg]];
          vs[pg] = a.kv_scales[2 * (size_t)x.id[pg] + 1];
        }
      }
      f32x16 z = logits<KV, D>(r, q);
      uint32_t seen = 0xffffu;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        z[i] *= a.scale_log2 * ks[i >> 3];
        if constexpr (kMasked) {
          const int pos = x.pos + 16 * (i >> 3) + key_of_reg<KV>(i & 7, hb);
          if (!(x.ok[i >> 3] && pos < row.limit)) z[i] = -INFINITY;
          if (!(x.ok[i >> 3] && pos < some)) seen &= ~(1u << i);
        }
      }
      weigh(st, z);
      add_values<KV, D, kMasked>(st, r, z, seen, vs);
    }
  };
  walk(std::false_type{});
  walk(std::true_type{});

  // ---- the four wavefronts' parts into one ------------------------------------
  st.sum += other_half(st.sum);
  if (lane < kRows) {
    s_m[wave][lane] = st.ref;
    s_l[wave][lane] = st.sum;
  }
  __syncthreads();
  for (int d0 = 0; d0 < D; d0 += DC) {
    if (d0) __syncthreads();
    float m = s_m[0][lane & 31];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) m = max_f(m, s_m[w][lane & 31]);
    const float f = exp2_fast(st.ref - m);
#pragma unroll
    for (int db = 0; db < DC / 32; ++db)
#pragma unroll
      for (int y = 0; y < 4; ++y)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          s_o[wave][lane & 31][32 * db + 8 * y + 4 * hb + e] = st.o[d0 / 32 + db][4 * y + e] * f;
    __syncthreads();
    for (int i = threadIdx.x; i < kRows * (DC / 4); i += 64 * kWaves) {
      const int rr = i / (DC / 4), d = i % (DC / 4) * 4;
      if (rr >= slot_rows || r0 + rr >= it.rows) continue;
      float mm = s_m[0][rr];
#pragma unroll
      for (int w = 1; w < kWaves; ++w) mm = max_f(mm, s_m[w][rr]);
      float l = 0.f;
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        l += s_l[w][rr] * exp2_fast(s_m[w][rr] - mm);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] += s_o[w][rr][d + e];
      }
      const float inv = l == 0.f ? 0.f : 1.f / l;
      const int64_t at = part0 + rr;
      f32x4 res;
#pragma unroll
      for (int e = 0; e < 4; ++e) res[e] = l == 0.f ? 0.f : o[e] * inv;
      *reinterpret_cast<f32x4 *>(a.part_o + at * D + d0 + d) = res;
      if (d0 + d == 0) a.part_lse[at] = l == 0.f ? -INFINITY : mm + log2f(l);
    }
  }
}

// ---------------------------------------------------------------------------
// merge: rows of (sequence, KV head) over the parts of its group and its own
// ---------------------------------------------------------------------------

template <int D>
__global__ __launch_bounds__(256) void merge_shared_kernel(SharedArgs a) {
  constexpr int D4 = D / 4;
  const int g = blockIdx.x % a.Hkv, b = blockIdx.x / a.Hkv;
  const int grp = group_of(a, b);
  const Unit own = seq_unit(a, b);
  Unit pre{0, 0, 0, 0};
  if (grp >= 0) pre = group_unit(a, grp);
  const PartsOf po = own.pages > 0 ? a.seq_parts[b] : PartsOf{0, 0, 0};
  const PartsOf pp = pre.pages > 0 ? a.group_parts[grp] : PartsOf{0, 0, 0};
  const int per = a.q_len * a.G;
  for (int i = threadIdx.x; i < per * D4; i += 256) {
    const int r = i / D4, d = i % D4 * 4;
    float m = kNoMax, l = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    auto add = [&](int64_t row0, int n, int rows, int rr) {
      const int rb = rr / rows;
      const int64_t at0 = row0 + (int64_t)(rb * a.Hkv + g) * n * rows + (rr - rb * rows);
      // (only with group offsets that do not ascend)
      if (row0 < 0 || n > a.grid || rr < 0 || at0 + (int64_t)(n - 1) * rows >= a.part_rows) return;
      for (int s = 0; s < n; ++s) {
        const int64_t at = at0 + (int64_t)s * rows;
        const float lse = a.part_lse[at];
        if (lse == -INFINITY) continue;              // no key seen
        const f32x4 v = *reinterpret_cast<const f32x4 *>(a.part_o + at * D + d);
        const float mm = max_f(m, lse);
        const float f = exp2_fast(m - mm), w = exp2_fast(lse - mm);
        m = mm;
        l = l * f + w;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          o[e] = (f == 0.f ? 0.f : o[e] * f) + (w == 0.f ? 0.f : v[e] * w);
      }
    };
    add(pp.row0, pp.n, a.shared_rows, (b - pre.seq0) * per + r);
    add(po.row0, po.n, a.own_rows, r);
    const int q = r / a.G;
    const int64_t row = ((int64_t)b * a.q_len + q) * a.Hq + g * a.G + (r - q * a.G);
    f32x4 res;
#pragma unroll
    for (int e = 0; e < 4; ++e) res[e] = l == 0.f ? 0.f : o[e] / l;
    *reinterpret_cast<f32x4 *>(a.out + row * D + d) = res;
    if (d == 0) a.lse[row] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
  }
}

template <int KV, int D>
void launch_d(const SharedArgs &a, hipStream_t s) {
  hipLaunchKernelGGL((attn_shared_kernel<KV, D>), dim3((unsigned)a.grid), dim3(64 * kWaves), 0, s, a);
  hipLaunchKernelGGL(merge_shared_kernel<D>, dim3((unsigned)(a.batch * a.Hkv)), dim3(256), 0, s, a);
}

template <int KV>
void launch_kv(const SharedArgs &a, hipStream_t s) {
  if (a.D == 64) launch_d<KV, 64>(a, s);
  else if (a.D == 128) launch_d<KV, 128>(a, s);
  else launch_d<KV, 256>(a, s);
}

}  // namespace

hipError_t launch_attn_shared(const SharedArgs &a, hipStream_t s) {
  if (a.kv_type == kF32) launch_kv<kF32>(a, s);
  else if (a.kv_type == kBF16) launch_kv<kBF16>(a, s);
  else launch_kv<kFP8>(a, s);
  return hipGetLastError();
}

}  // namespace kap

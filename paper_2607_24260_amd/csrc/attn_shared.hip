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
// A workgroup takes a split of a group's shared pages with up to 32 WR rows: WR
// wavefronts with 32 rows each, as many wavefronts as that leaves by different
// keys. From WR = 2 on the pages go through LDS, so that each is read once per
// workgroup, in operand blocks of 1 KB laid out as the lanes multiply them; fp8
// codes are widened on the way in. With WR = 1, and for a sequence's own pages (a
// wavefront by itself: unit, row block, KV head and split), operands go straight
// from memory to the lane's registers, the next step's on the way while this one
// is multiplied.
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

// Work item of a wavefront. A step of a group's shared pages costs a.shared_cost, one
// of a sequence's own a.own_cost (a wavefront's share of a workgroup's time). C is
// what a workgroup gets; shared pages are split into parts of up to C, a workgroup
// each, a sequence's own into parts of up to C over the wavefronts of a workgroup, a
// wavefront each. The last part of a unit is not full, by one half on average and by
// more in a unit shorter than C: C is the cost of all units over the workgroups
// wanted less those, so that what runs at once is filled and no few parts are left to
// run after it. Parts are numbered group by group, then sequence by sequence. There
// are at most total / C, so at most `target`, workgroups plus one part per (unit, row
// block, head): the grid. The sums are float32, their rounding well inside the slack
// taken of C: every wavefront of the launch finds the same C, from the same operations.
template <int WAVES>
__device__ bool shared_map(const SharedArgs &a, int w, int wave, Item &it) {
  const int lane = threadIdx.x & 63;
  auto steps_of = [](const Unit &u) { return (u.pages + 1) / 2; };
  auto blocks_of = [&](const Unit &u, bool shared) {
    const int br = shared ? a.shared_rows : a.own_rows;
    return div_small(u.rows + br - 1, br);
  };
  auto unit_of = [&](bool shared, int i) {
    const int n = shared ? a.num_groups : a.batch;
    if (i >= n) return Unit{0, 0, 0, 0};
    return shared ? group_unit(a, i) : seq_unit(a, i);
  };
  Unit first[2];                               // of the first 64, kept for the later passes
  first[0] = unit_of(true, lane);
  first[1] = unit_of(false, lane);
  // f(cost, row blocks, shared) of all units, the sum over the lanes
  auto sum = [&](auto f) {
    auto of = [&](const Unit &u, bool shared) {
      return f((float)steps_of(u) * (float)(shared ? a.shared_cost : a.own_cost),
               (float)(u.pages > 0 ? blocks_of(u, shared) : 0), shared);
    };
    float x = of(first[0], true) + of(first[1], false);
    for (int i0 = 64; i0 < a.num_groups; i0 += 64) x += of(unit_of(true, i0 + lane), true);
    for (int i0 = 64; i0 < a.batch; i0 += 64) x += of(unit_of(false, i0 + lane), false);
    return wave_sum(x) * (float)a.Hkv;
  };
  const float total = sum([](float cost, float blocks, bool) { return cost * blocks; });
  const float per = (float)a.target / fmaxf(total, 1.f);
  const float unfilled = sum([&](float cost, float blocks, bool shared) {
    const float full = cost * per * (shared ? 1.f : (float)WAVES);   // parts, were they all full
    return fmaxf(0.5f, 1.f - full) * blocks * (shared ? 1.f : 1.f / WAVES);
  });
  const float wanted = fmaxf((float)a.target - unfilled, 0.5f * a.target);
  const float most = fmaxf(total * 1.0001f / wanted, (float)a.least);
  const int len[2] = {                         // steps of a part
      (int)fminf(ceilf(most / a.shared_cost), 1e9f),
      max((int)fminf(ceilf(most / (a.own_cost * WAVES)), 1e9f), a.own_least)};
  int base = 0;
  for (int kind = 0; kind < 2; ++kind) {
    const bool shared = kind == 0;
    const int n = shared ? a.num_groups : a.batch;
    const int slot_rows = shared ? a.shared_rows : a.own_rows;
    const int64_t start = shared ? 0 : a.own_base;
    if (!shared) {                             // parts are wavefronts' from here on
      w = (w - base) * WAVES + wave;
      base = 0;
    }
    for (int i0 = 0; i0 < n; i0 += 64) {
      const Unit u = i0 == 0 ? first[kind] : unit_of(shared, i0 + lane);
      const int rb = blocks_of(u, shared);
      const int parts = div_small(steps_of(u) + len[kind] - 1, len[kind]);
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
        const int e = base + __builtin_amdgcn_readlane(excl, l);
        it.row0 = start + (int64_t)e * slot_rows;
        const int off = w - e;
        const int block = div_small(off, it.n_split);
        it.split = off - block * it.n_split;
        it.rb = div_small(block, a.Hkv);
        it.g = block - it.rb * a.Hkv;
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

// The same in registers ...
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

// ... and in LDS: blocks of 64 lanes' 16 bytes, K's and then V's.
template <int KV, int D>
struct Tile {
  static constexpr int kBytes = 2 * operands<KV, D>() * 1024;
  const u32x4 *at;                             // of this lane
  __device__ u32x4 key(int c) const { return at[c * 64]; }
  __device__ u32x4 value(int y, int db) const {
    return at[(operands<KV, D>() + y * (D / 32) + db) * 64];
  }
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

// Moves the reference above a step's logits (c z: in powers of two, c >= 0).
template <int D>
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
      for (int i = 0; i < 16; ++i) st.o[db][i] *= f;
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
    u32x4 hi, lo, sees;
    if constexpr (KV != kF32) {
      float p[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) p[i] = KV == kFP8 ? w[8 * y + i] * vs[y] : w[8 * y + i];
      split8(p, hi, lo);
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
  return RowOf{((int64_t)b * a.q_len + i) * a.Hq + it.g * a.G + (rr - i * a.G),
               max(0, min(a.seq_lens[b], a.max_pages * kPage) - a.q_len + i + 1)};
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
  int cur, next, k0, first, stride;
  __device__ int fetch(const Walk &w, int k) const {
    const int lane = threadIdx.x & 63, e = 2 * (first + (k + (lane >> 1)) * stride) + (lane & 1);
    return w.table[min(e, max(w.pages - 1, 0))];
  }
  __device__ PageIds(const Walk &w, int first_, int stride_) : k0(0), first(first_), stride(stride_) {
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
// plain: what positions allow, if all the pages up to there are in the pool (the
// lanes of `n` threads look at them).
__device__ __forceinline__ bool pages_fine(const SharedArgs &a, const Walk &w, int thread, int n) {
  bool fine = true;
  for (int i = 2 * w.s0 + thread; i < 2 * w.plain; i += n) fine &= in_pool(a, w.table[i]);
  return fine;
}
__device__ __forceinline__ int plain_by_position(const Walk &w) {
  return max(w.s0, min(min(w.s1, w.pages / 2), (w.all / kPage - w.page0) / 2));
}

// Raw logits to powers of two, up to the factor that is returned (not negative:
// the sign of sm_scale is in Q). MASKED: keys that a row does not see to -inf.
template <int KV, bool MASKED>
__device__ __forceinline__ float scale_logits(const SharedArgs &a, const Walk &w, f32x16 &z,
                                              uint32_t &seen, int s, const bool (&ok)[2], int limit,
                                              const float (&ks)[2]) {
  const int hb = (threadIdx.x & 63) >> 5;
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
                                          const float (&vs)[2]) {
  f32x16 z = logits<KV, D>(src, q);
  uint32_t seen;
  const float c = scale_logits<KV, MASKED>(a, w, z, seen, s, ok, limit, ks);
  move_reference(st, z, c);
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

// Steps first, first + stride, .. below w.s1, operands from memory.
template <int KV, int D>
__device__ __forceinline__ void walk_memory(State<D> &st, const SharedArgs &a, const Walk &w,
                                            const Queries<KV, D> &q, int g, int first, int stride,
                                            int limit) {
  const int lane = threadIdx.x & 63;
  if (first >= w.s1) return;
  PageIds ids(w, first, stride);
  int k = 0;
  auto step = [&](int i) { return first + i * stride; };
  if constexpr (KV != kF32 || D < 256) {
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
        const float c = scale_logits<KV, false>(a, w, z, seen, step(k), fine, limit, ks);
        move_reference(st, z, c);
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
    take_step<KV, D, true>(st, a, w, q, Pages<KV, D>(a, x.id, g, lane), step(k), x.ok, limit, ks, vs);
  }
}

// ---------------------------------------------------------------------------
// shared pages through LDS
// ---------------------------------------------------------------------------

// A stage is WK = WAVES / WR tiles of 32 keys. Half of the wavefronts fetch K,
// half V: each a run of one tile's blocks, into registers, several stages ahead of
// the LDS buffer they go to. Stage i multiplies K of i + 1 and V of i, so that the
// matrix unit has the next logits to work on while the vector unit turns these
// into weights (all wavefronts do the same between two barriers: without that a
// stage of 256 rows took 3500 cycles, 1536 of them matrix instructions and about as
// many vector instructions). Of K and of V there are two buffers, and one barrier a
// stage: a buffer is written again only after all wavefronts have passed the
// barrier that follows its last use.
template <int KV, int D, int WR>
struct Staging {
  static constexpr int kWaves = waves_of(KV, D), kTiles = kWaves / WR, kHalf = kWaves / 2;
  // 1 KB loads of a tile's K (or V), and of a wavefront in a stage
  static constexpr int kLoads = KV == kFP8 ? operands<KV, D>() / 2 : operands<KV, D>();
  static constexpr int kMine = kLoads * kTiles < kHalf ? 1 : kLoads * kTiles / kHalf;
  static constexpr int kBusy = kLoads * kTiles / kMine;   // of a half; any others fetch the same
  static constexpr int kAhead = kMine >= 8 ? 1 : (kMine >= 4 ? 2 : 4);   // stages
  static constexpr int kStage = kTiles * Tile<KV, D>::kBytes;
  static constexpr int kScales = KV == kFP8 ? 4 * kTiles * 4 * 4 : 0;   // of four stages
  static constexpr int kBytes = 2 * kStage + kScales;
};

// A stage of one wavefront: weights of the logits z of tile `now` and its values,
// and z of tile `next`. Operands are read from LDS a group of four ahead of the
// matrix instructions that take them, in regions that the scheduler may not cross
// (left alone, it reads each operand right before it is multiplied: most of a stage
// was waiting for LDS), and the vector instructions are shared out over them.
template <int KV, int D, bool MASKED>
__device__ __forceinline__ void staged_step(State<D> &st, f32x16 &z, const SharedArgs &a,
                                            const Walk &walk, const Queries<KV, D> &q,
                                            const Tile<KV, D> &now, const Tile<KV, D> &next, int s,
                                            const bool (&ok)[2], int limit, const float (&ks)[2],
                                            const float (&vs)[2]) {
  constexpr int K = operands<KV, D>(), DB = D / 32;
  constexpr int kGroup = DB < 4 ? DB : 4;                  // operands of a group
  constexpr int kQk = K / kGroup, kPv = DB / kGroup;       // groups: K's, V's of a page
  constexpr int kGroups = kQk + 2 * kPv;
  u32x4 op[2][kGroup];
  auto read = [&](int g, u32x4 (&to)[kGroup]) {
#pragma unroll
    for (int i = 0; i < kGroup; ++i) {
      if (g < kQk) to[i] = next.key(g * kGroup + i);
      else to[i] = now.value((g - kQk) / kPv, (g - kQk) % kPv * kGroup + i);
    }
  };
  read(0, op[0]);
  __builtin_amdgcn_sched_barrier(0);
  uint32_t seen, wild = 0;
  const float c = scale_logits<KV, MASKED>(a, walk, z, seen, s, ok, limit, ks);
  move_reference(st, z, c);
  __builtin_amdgcn_sched_barrier(0);
  f32x16 z1 = zero16();
  u32x4 hi, lo, sees;
  auto weigh_page = [&](int y) {
#pragma unroll
    for (int i = 8 * y; i < 8 * y + 8; ++i) {
      z[i] = exp2_fast(fmaf(z[i], c, -st.ref));
      st.sum += z[i];
    }
  };
  u32x4 hi1, lo1;
  auto split_page = [&](int y, u32x4 &h, u32x4 &l) {
    float p[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = KV == kFP8 ? z[8 * y + i] * vs[y] : z[8 * y + i];
    split8(p, h, l);
  };
#pragma unroll
  for (int g = 0; g < kGroups; ++g) {
    if (g + 1 < kGroups) read(g + 1, op[(g + 1) & 1]);
    if (g < kQk) {
#pragma unroll
      for (int i = 0; i < kGroup; ++i) z1 = mfma(op[g & 1][i], q.at(g * kGroup + i), z1);
      if (g == 0) weigh_page(0);
      if (g == kQk - 1) {
        split_page(0, hi, lo);
        weigh_page(1);
      }
    } else {
      const int y = (g - kQk) / kPv, db0 = (g - kQk) % kPv * kGroup;
      if constexpr (MASKED) sees = seen_words<KV>(seen, y);
#pragma unroll
      for (int i = 0; i < kGroup; ++i) {
        u32x4 v = op[g & 1][i];
        if constexpr (MASKED) {
          v &= sees;
          const u32x4 m = wild_words<KV>(v);
          wild |= m[0] | m[1] | m[2] | m[3];
          v &= ~m;
        }
        st.o[db0 + i] = mfma(v, y ? hi1 : hi, st.o[db0 + i]);
        st.o[db0 + i] = mfma(v, y ? lo1 : lo, st.o[db0 + i]);
      }
      if (g == kQk) split_page(1, hi1, lo1);
    }
    __builtin_amdgcn_sched_barrier(0);
  }
  if constexpr (MASKED)
    if (__any(wild != 0u)) add_classes<KV, D>(st, now, z, seen);
  z = z1;
}

template <int KV, int D, int WR>
__device__ __forceinline__ void walk_staged(State<D> &st, const SharedArgs &a, const Walk &w,
                                            const Queries<KV, D> &q, int g, int limit, bool idle,
                                            char *smem) {
  using S = Staging<KV, D, WR>;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kw = wave / WR;                    // tile of a stage this wavefront multiplies
  // what it fetches
  const bool is_v = wave >= S::kHalf;
  const int load0 = wave % S::kBusy * S::kMine, tile = load0 / S::kLoads, c0 = load0 % S::kLoads;
  const bool has_scales = KV == kFP8 && !is_v && c0 == 0;
  constexpr size_t kPageTile = Pages<KV, D>::kTile;
  const char *const k_pages = static_cast<const char *>(a.k_pages);
  const char *const v_pages = static_cast<const char *>(a.v_pages);
  const char *const pages = is_v ? v_pages : k_pages;
  u32x4 raw[S::kAhead][S::kMine];
  float raw_scale[S::kAhead];
  PageIds ids(w, w.s0 + tile, S::kTiles);
  const int stages = (w.s1 - w.s0 + S::kTiles - 1) / S::kTiles;
  const int plain = (w.plain - w.s0) / S::kTiles;

  auto fetch = [&](int stage, int slot) __attribute__((always_inline)) {
    const bool live = stage < stages;
    const Step x = ids.at(a, w, stage);
    const int id0 = x.id[0], id1 = x.id[1];
    if constexpr (KV == kFP8) {
#pragma unroll
      for (int t = 0; t < S::kMine; ++t) {
        const int c = c0 + t, pg = c / (D / 64), part = c % (D / 64);
        const int id = pg ? id1 : id0;
        raw[slot][t] = *reinterpret_cast<const u32x4 *>(
            pages + ((size_t)id * a.Hkv + g) * kPageTile + (live ? part * 1024 + lane * 16 : 0));
      }
      raw_scale[slot] = a.kv_scales[2 * (size_t)(lane & 2 ? id1 : id0) + (lane & 1)];
    } else {
      const Pages<KV, D> p(a, x.id, g, lane, live);
#pragma unroll
      for (int t = 0; t < S::kMine; ++t) {
        const int c = c0 + t;
        raw[slot][t] = is_v ? p.raw_value(c / (D / 32), c % (D / 32)).x : p.raw_key(c).x;
      }
    }
  };
  auto place = [&](int stage, int slot) __attribute__((always_inline)) {
    u32x4 *to = reinterpret_cast<u32x4 *>(smem + (stage & 1) * S::kStage + tile * Tile<KV, D>::kBytes) +
                (is_v ? operands<KV, D>() * 64 : 0);
#pragma unroll
    for (int t = 0; t < S::kMine; ++t) {
      const int c = c0 + t;
      if constexpr (KV == kFP8) {
        const int pg = c / (D / 64), part = c % (D / 64);
        const u32x4 lo = widen8(u32x2{raw[slot][t][0], raw[slot][t][1]});
        const u32x4 hi = widen8(u32x2{raw[slot][t][2], raw[slot][t][3]});
        if (is_v) {                            // dim 64 part + lane: its keys 0..7 and 8..15
          u32x4 *at = to + (pg * (D / 32) + 2 * part + (lane >> 5)) * 64 + (lane & 31);
          at[0] = lo;
          at[32] = hi;
        } else {                               // chunk 8 part + lane / 8, two tokens
          const int chunk = 8 * part + (lane >> 3), tok = 2 * (lane & 7);
          u32x4 *at = to + (chunk >> 1) * 64 + (chunk & 1) * 32 + 16 * pg;
          at[key_of_row<KV>(tok)] = lo;
          at[key_of_row<KV>(tok + 1)] = hi;
        }
      } else {
        to[c * 64 + lane] = raw[slot][t];
      }
    }
    if (has_scales && lane < 4)
      reinterpret_cast<float *>(smem + 2 * S::kStage)[((stage & 3) * S::kTiles + tile) * 4 + lane] =
          raw_scale[slot];
  };

  // K runs a stage ahead of V: its wavefronts' slot of stage i holds stage i + 1.
  const int lead = is_v ? 0 : 1;
  auto tile_at = [&](int stage) {
    return Tile<KV, D>{reinterpret_cast<const u32x4 *>(smem + (stage & 1) * S::kStage +
                                                       kw * Tile<KV, D>::kBytes) + lane};
  };
  if (lead) {
    fetch(0, 0);
    place(0, 0);
  }
#pragma unroll
  for (int u = 0; u < S::kAhead; ++u)
    fetch(u + lead, u);
  __syncthreads();
  f32x16 z = zero16();
  if (!idle) z = logits<KV, D>(tile_at(0), q);
  int stage0 = 0;
  auto walk = [&](auto masked, int end) __attribute__((always_inline)) {
    constexpr bool kMasked = decltype(masked)::value;
    // (slots are numbered from the walk's first stage on, which is a multiple of kAhead)
    for (; stage0 < end; stage0 += S::kAhead) {
#pragma unroll
      for (int u = 0; u < S::kAhead; ++u) {
        const int stage = stage0 + u;
        if (kMasked && stage >= end) break;
        place(stage + lead, u);
        __syncthreads();
        fetch(stage + lead + S::kAhead, u);
        if (idle) continue;
        float ks[2] = {1.f, 1.f}, vs[2] = {1.f, 1.f};
        if constexpr (KV == kFP8) {
          const f32x4 sc = *reinterpret_cast<const f32x4 *>(
              smem + 2 * S::kStage + ((stage & 3) * S::kTiles + kw) * 16);
          ks[0] = sc[0];
          vs[0] = sc[1];
          ks[1] = sc[2];
          vs[1] = sc[3];
        }
        const int s = w.s0 + stage * S::kTiles + kw;
        bool ok[2] = {true, true};
        if constexpr (kMasked) {               // (few stages: ids are read again)
#pragma unroll
          for (int pg = 0; pg < 2; ++pg)
            ok[pg] = s < w.s1 && 2 * s + pg < w.pages && in_pool(a, w.table[2 * s + pg]);
        }
        // (past the last stage: what the buffer holds, for nothing)
        staged_step<KV, D, kMasked>(st, z, a, w, q, tile_at(stage), tile_at(stage + 1), s, ok, limit,
                                    ks, vs);
      }
    }
  };
  walk(std::false_type{}, plain / S::kAhead * S::kAhead);
  walk(std::true_type{}, stages);
  __syncthreads();
}

// ---------------------------------------------------------------------------
// the kernel
// ---------------------------------------------------------------------------

template <int KV, int D, int WR>
struct Layout {
  static constexpr int kWaves = waves_of(KV, D);
  // the wavefronts' parts, 32 dims at a time: [wave][row][32 dims + 4]
  static constexpr int kPart = kRows * 36 * 4;
  static constexpr int kStaged = [] {
    if constexpr (WR > 1) return Staging<KV, D, WR>::kBytes;
    else return 0;
  }();
  static constexpr int kWalk = kStaged > kWaves * kPart ? kStaged : kWaves * kPart;
  static constexpr int kBytes =
      kWalk + (q_in_lds<KV, D>() ? kWaves * operands<KV, D>() * 1024 : 0);
};

template <int KV, int D, int WR>
__global__ __launch_bounds__(64 * waves_of(KV, D))
__attribute__((amdgpu_waves_per_eu(waves_of(KV, D) / 4)))
void attn_shared_kernel(SharedArgs a) {
  constexpr int kWaves = waves_of(KV, D), kTiles = kWaves / WR;
  __shared__ __align__(16) char smem[Layout<KV, D, WR>::kBytes];
  __shared__ float s_m[kWaves][kRows], s_l[kWaves][kRows];
  __shared__ int s_all, s_some, s_bad;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int hb = lane >> 5;
  if (threadIdx.x == 0) {
    s_all = 0x7fffffff;
    s_some = 0;
    s_bad = 0;
  }
  Item it;
  if (!shared_map<kWaves>(a, blockIdx.x, wave, it)) return;   // (a shared part: all wavefronts)
  const int slot_rows = it.shared ? a.shared_rows : a.own_rows;
  const int64_t part0 =
      it.row0 + ((int64_t)(it.rb * a.Hkv + it.g) * it.n_split + it.split) * slot_rows;
  // (group offsets that do not ascend)
  if (part0 + slot_rows > (it.shared ? a.own_base : a.part_rows)) return;
  if (it.rb == 0 && it.g == 0 && it.split == 0 && (it.shared ? threadIdx.x == 0 : lane == 0))
    (it.shared ? a.group_parts : a.seq_parts)[it.unit] = PartsOf{it.row0, it.n_split, 0};

  // ---- rows ---------------------------------------------------------------------
  const int rw = it.shared ? wave % WR : 0;
  const int r0 = it.rb * slot_rows + rw * kRows;        // of the unit
  const int in_block = rw * kRows + (lane & 31);
  const RowOf row = row_of(a, it, in_block < slot_rows ? it.rb * slot_rows + in_block : it.rows);
  Queries<KV, D> q;
  {
    constexpr int kBytes = KV == kF32 ? 4 : 2;
    const char *p = static_cast<const char *>(a.q) + (row.q < 0 ? 0 : row.q) * D * kBytes + hb * 16;
    u32x4 *lds = reinterpret_cast<u32x4 *>(smem + Layout<KV, D, WR>::kWalk) +
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
  Walk w;
  w.table = a.table + (size_t)it.seq0 * a.stride + it.page0;
  w.page0 = it.page0;
  w.pages = it.pages;
  const int steps = (it.pages + 1) / 2;
  w.s0 = (int)((long long)steps * it.split / it.n_split);
  w.s1 = (int)((long long)steps * (it.split + 1) / it.n_split);
  int all = row.q < 0 ? 0x7fffffff : row.limit, some = row.limit;
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) {
    all = min(all, __shfl_xor(all, o, 64));
    some = max(some, __shfl_xor(some, o, 64));
  }
  State<D> st;
#pragma unroll
  for (int db = 0; db < D / 32; ++db) st.o[db] = zero16();
  st.ref = kNoMax;
  st.sum = 0.f;

  if (!it.shared) {
    // ---- a wavefront by itself ----------------------------------------------------
    w.all = __builtin_amdgcn_readfirstlane(all);
    w.some = __builtin_amdgcn_readfirstlane(some);
    w.plain = plain_by_position(w);
    if (__any(!pages_fine(a, w, lane, 64))) w.plain = w.s0;
    walk_memory<KV, D>(st, a, w, q, it.g, w.s0, 1, row.limit);
    st.sum += other_half(st.sum);
    const int rr = lane & 31;
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

  // ---- a workgroup --------------------------------------------------------------
  __syncthreads();
  if (lane == 0) {
    atomicMin(&s_all, all);
    atomicMax(&s_some, some);
  }
  __syncthreads();
  w.all = __builtin_amdgcn_readfirstlane(s_all);
  w.some = __builtin_amdgcn_readfirstlane(s_some);
  w.plain = plain_by_position(w);
  if (!pages_fine(a, w, threadIdx.x, 64 * kWaves)) s_bad = 1;
  __syncthreads();
  if (__builtin_amdgcn_readfirstlane(s_bad)) w.plain = w.s0;
  if constexpr (WR == 1) {
    walk_memory<KV, D>(st, a, w, q, it.g, w.s0 + wave, kWaves, row.limit);
  } else {
    walk_staged<KV, D, WR>(st, a, w, q, it.g, row.limit, r0 >= it.rows, smem);
  }
  st.sum += other_half(st.sum);
  if (lane < kRows) {
    s_m[wave][lane] = st.ref;
    s_l[wave][lane] = st.sum;
  }
  __syncthreads();
  // the wavefronts with other keys of the same rows: wave % WR + WR t
  float *part = reinterpret_cast<float *>(smem);
  float m = s_m[rw][lane & 31];
#pragma unroll
  for (int t = 1; t < kTiles; ++t) m = max_f(m, s_m[rw + WR * t][lane & 31]);
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
          for (int e = 0; e < 4; ++e) v[e] = st.o[d][4 * y + e] * f;
          *reinterpret_cast<f32x4 *>(part + (wave * kRows + (lane & 31)) * 36 + 8 * y + 4 * hb) = v;
        }
      }
    __syncthreads();
    for (int i = threadIdx.x; i < WR * kRows * 8; i += 64 * kWaves) {
      const int rr = i >> 3, d = (i & 7) * 4, rg = rr / kRows, rl = rr % kRows;
      if (rr >= slot_rows || it.rb * slot_rows + rr >= it.rows) continue;
      float mm = s_m[rg][rl];
#pragma unroll
      for (int t = 1; t < kTiles; ++t) mm = max_f(mm, s_m[rg + WR * t][rl]);
      float l = 0.f;
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int t = 0; t < kTiles; ++t) {
        const int v = rg + WR * t;
        l += s_l[v][rl] * exp2_fast(s_m[v][rl] - mm);
        const f32x4 x = *reinterpret_cast<const f32x4 *>(part + (v * kRows + rl) * 36 + d);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] += x[e];
      }
      const float inv = l == 0.f ? 0.f : 1.f / l;
      f32x4 res;
#pragma unroll
      for (int e = 0; e < 4; ++e) res[e] = l == 0.f ? 0.f : o[e] * inv;
      *reinterpret_cast<f32x4 *>(a.part_o + (part0 + rr) * D + 32 * db + d) = res;
      if (db == 0 && d == 0) a.part_lse[part0 + rr] = l == 0.f ? -INFINITY : mm + log2f(l);
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
  const int g = blockIdx.x % a.Hkv, b = blockIdx.x / a.Hkv;
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
  add(pp.row0, pp.n, a.shared_rows, (b - pre.seq0) * per + r);
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
  const dim3 grid((unsigned)a.grid), block(64 * kWaves);
  const int wr = a.shared_rows / kRows;
  if (wr == 1) hipLaunchKernelGGL((attn_shared_kernel<KV, D, 1>), grid, block, 0, s, a);
  if constexpr (KV != kF32) {
    if (wr == 2) hipLaunchKernelGGL((attn_shared_kernel<KV, D, 2>), grid, block, 0, s, a);
    if (wr == 4) hipLaunchKernelGGL((attn_shared_kernel<KV, D, 4>), grid, block, 0, s, a);
    if constexpr (kWaves == 8)
      if (wr == 8) hipLaunchKernelGGL((attn_shared_kernel<KV, D, 8>), grid, block, 0, s, a);
  }
  const int items = a.q_len * a.G * (D / 4);
  hipLaunchKernelGGL(merge_shared_kernel<D>,
                     dim3((unsigned)(a.batch * a.Hkv), (unsigned)((items + kItems - 1) / kItems)),
                     dim3(kItems * kShares), 0, s, a);
}

template <int KV>
void launch_kv(const SharedArgs &a, hipStream_t s) {
  if (a.D == 64) launch_d<KV, 64>(a, s);
  else if (a.D == 128) launch_d<KV, 128>(a, s);
  else launch_d<KV, 256>(a, s);
}

}  // namespace

// Wavefronts with rows of their own: enough for a group's rows, of the numbers
// there are kernels for. float32 takes one: its matrix instructions are what such
// a call waits for (32 rows and keys of 128 dims: 8192 cycles of them for 32 KB),
// and row blocks that read the same pages again get them from the caches.
int shared_row_waves(int kv_type, int D, long long rows) {
  if (kv_type == kF32) return 1;
  int wr = 1;
  while (wr < waves_of(kv_type, D) && rows > (long long)wr * kRows) wr *= 2;
  return wr;
}
int shared_waves(int kv_type, int D) { return waves_of(kv_type, D); }

hipError_t launch_attn_shared(const SharedArgs &a, hipStream_t s) {
  if (a.kv_type == kF32) launch_kv<kF32>(a, s);
  else if (a.kv_type == kBF16) launch_kv<kBF16>(a, s);
  else launch_kv<kFP8>(a, s);
  return hipGetLastError();
}

}  // namespace kap

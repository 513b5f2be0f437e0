// Attention of ragged chunks of new tokens -- from one token a sequence to whole
// prompts -- over the paged cache, causal, with a sliding window and sinks or without.
//
// The rows of a (sequence, KV head) are its new tokens times the query heads of the
// KV head, token by token. A wavefront holds 32 rows and walks 32 keys (two pages) a
// step (attn_tiles.h). Rows see positions lo <= t < hi and t < sinks; a block of rows
// walks the steps that hold its sinks, then those from its lowest lo to its highest hi.
#include "attn_tiles.h"
#include "block_scan.h"

#include <algorithm>

namespace kap {
namespace {

constexpr int kRows = 32;                      // of a wavefront
constexpr int kKeys = 32;                      // of a step
constexpr int waves_of(int kv, int D) { return chunk_waves(kv, D); }

// ---------------------------------------------------------------------------
// work map
// ---------------------------------------------------------------------------

// A sequence's part in a call.
struct Seq {
  int q0, n, len;    // first row of q, new tokens, length
  int rows;          // n * G
  bool tall;         // more rows than a few wavefronts': workgroups take them
  int block, blocks; // rows of a block, blocks
};

__device__ __forceinline__ Seq seq_of(const ChunkArgs &a, int b, int tall_rows) {
  Seq s;
  s.q0 = clamp_to(a.q_offsets[b], 0, a.num_tokens);
  s.n = clamp_to(a.q_offsets[b + 1], s.q0, a.num_tokens) - s.q0;
  s.len = clamp_to(a.seq_lens[b], 0, a.max_len);
  s.rows = s.n * a.G;
  s.tall = s.rows > a.few_rows;
  s.block = s.tall ? tall_rows : kRows;
  s.blocks = div_small(s.rows + s.block - 1, s.block);
  return s;
}

// Steps that rows [r0, r1) of a sequence walk: the first `sinks` of them, then those
// from `from` on.
struct Range {
  int sinks, from, steps;
};
__device__ __forceinline__ Range range_of(const ChunkArgs &a, const Seq &s, int r0, int r1) {
  const int p0 = s.len - s.n + div_small(r0, a.G), p1 = s.len - s.n + div_small(r1 - 1, a.G);
  Range r;
  const int hi = max(0, p1 + 1);
  const int lo = a.window > 0 ? max(0, p0 - a.window + 1) : 0;
  r.from = min(lo, hi) / kKeys;
  r.sinks = min((min(a.sinks, hi) + kKeys - 1) / kKeys, r.from);
  r.steps = r.sinks + (hi + kKeys - 1) / kKeys - r.from;
  return r;
}
__device__ __forceinline__ Range block_range(const ChunkArgs &a, const Seq &s, int block) {
  return range_of(a, s, block * s.block, min((block + 1) * s.block, s.rows));
}

// The map: what a part of a tall sequence's block, and of another's, walks at most;
// their number; blocks to merge. Then, per sequence, sums before it: of tall parts, of
// others, of blocks to merge; its splits and the first row of its partials.
enum MapHead { kMapTall, kMapFew, kMapMerge, kMapHead = 4 };
struct MapOf {
  int32_t *head, *tall, *few, *merge, *splits;
  int64_t *row0;
};
__device__ __forceinline__ MapOf map_of(const ChunkArgs &a) {
  MapOf m;
  m.row0 = reinterpret_cast<int64_t *>(a.map);
  m.head = reinterpret_cast<int32_t *>(m.row0 + a.batch);
  m.tall = m.head + kMapHead;
  m.few = m.tall + a.batch;
  m.merge = m.few + a.batch;
  m.splits = m.merge + a.batch;
  return m;
}

template <int WAVES>
__global__ __launch_bounds__(kScanThreads) void chunk_plan_kernel(ChunkArgs a) {
  __shared__ long long s_scan[4][kScanWaves];
  const MapOf m = map_of(a);
  constexpr int kTall = kRows * WAVES;
  // the steps there are, in those of a workgroup with a tall block
  long long sum = 0;
  for (int b = threadIdx.x; b < a.batch; b += kScanThreads) {
    const Seq s = seq_of(a, b, kTall);
    if (s.blocks == 0) continue;
    const long long steps =
        (block_range(a, s, 0).steps + block_range(a, s, s.blocks - 1).steps + 1) / 2;
    sum += steps * s.blocks * (s.tall ? a.tall_cost : a.few_cost);
  }
  {
    const long long x[1] = {sum};
    long long incl[1], total[1];
    scan(x, incl, total, s_scan);
    sum = total[0] * a.Hkv;
  }
  // of a part, were all alike
  const long long per = max(1ll, (sum + a.target - 1) / a.target);
  const int tall_len = (int)min(max((per + a.tall_cost - 1) / a.tall_cost, (long long)a.tall_least), 1ll << 30);
  const int few_len =
      (int)min(max((per + WAVES * a.few_cost - 1) / (WAVES * a.few_cost), (long long)a.few_least), 1ll << 30);
  long long tall = 0, few = 0, merge = 0, rows = 0;
  for (int b0 = 0; b0 < a.batch; b0 += kScanThreads) {
    const int b = b0 + threadIdx.x;
    const bool in = b < a.batch;
    Seq s{};
    int splits = 0;
    long long slots = 0;
    if (in) {
      s = seq_of(a, b, kTall);
      if (s.blocks > 0) {
        const int most = max(block_range(a, s, 0).steps, block_range(a, s, s.blocks - 1).steps);
        const int len = s.tall ? tall_len : few_len;
        splits = max(1, div_small(most + len - 1, len));
        if (splits > 1) slots = (long long)splits * s.blocks * a.Hkv * min(s.block, s.rows);
      }
    }
    {
      const long long x[1] = {slots};
      long long incl[1], total[1];
      scan(x, incl, total, s_scan);
      if (slots > 0 && rows + incl[0] > a.part_rows) splits = 1;   // no room for its partials
      if (in) m.row0[b] = rows + incl[0] - slots;
      rows += total[0];
    }
    const long long parts = (long long)s.blocks * splits * a.Hkv;
    const long long x[3] = {s.tall ? parts : 0, s.tall ? 0 : parts,
                            splits > 1 ? (long long)s.blocks * a.Hkv : 0};
    long long incl[3], total[3];
    scan(x, incl, total, s_scan);
    if (in) {
      m.tall[b] = (int)(tall + incl[0] - x[0]);
      m.few[b] = (int)(few + incl[1] - x[1]);
      m.merge[b] = (int)(merge + incl[2] - x[2]);
      m.splits[b] = splits;
    }
    tall += total[0];
    few += total[1];
    merge += total[2];
  }
  if (threadIdx.x == 0) {
    m.head[kMapTall] = (int)tall;
    m.head[kMapFew] = (int)few;
    m.head[kMapMerge] = (int)merge;
  }
}

// The last of the sequences whose sum is at most w (by a whole wavefront).
__device__ __forceinline__ int find(const int32_t *first, int n, int w, int lane) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int step = (hi - lo + 63) / 64, i = lo + lane * step;
    const unsigned long long hit = __ballot(i < hi && first[min(i, hi - 1)] <= w);
    lo += (__popcll(hit) - 1) * step;
    hi = min(lo + step, hi);
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

// What a wavefront does: rows [r0, r1) of a sequence's KV head g over steps [j0, j1) of
// a range, and where the result goes (part < 0: out).
struct Item {
  Seq s;
  int b, g, r0, r1;
  Range r;
  int j0, j1;
  int own0, own1;    // of which these rows see something in [own0, own1) (tall: of the block's)
  bool tall;
  int last_rows;     // where the block's last wavefront with rows starts
  int64_t part;
};

template <int WAVES>
__device__ bool item_of(const ChunkArgs &a, int w, int wave, int lane, Item &it) {
  const MapOf m = map_of(a);
  constexpr int kTall = kRows * WAVES;
  const bool tall = w < m.head[kMapTall];
  if (!tall) {
    w = (w - m.head[kMapTall]) * WAVES + wave;
    if (w >= m.head[kMapFew]) return false;
  }
  const int32_t *first = tall ? m.tall : m.few;
  it.b = find(first, a.batch, w, lane);
  it.s = seq_of(a, it.b, kTall);
  const int splits = m.splits[it.b], off = w - first[it.b];
  if (off < 0 || splits < 1) return false;     // (offsets that do not ascend)
  int block, split;
  if (tall) {                                  // the longest first; KV heads share out the XCDs
    const int at = div_small(off, a.Hkv);
    it.g = off - at * a.Hkv;
    block = div_small(at, splits);
    split = at - block * splits;
    block = it.s.blocks - 1 - block;
  } else {
    const int at = div_small(off, splits);
    split = off - at * splits;
    block = div_small(at, a.Hkv);
    it.g = at - block * a.Hkv;
  }
  if (block < 0 || block >= it.s.blocks) return false;
  it.r = block_range(a, it.s, block);
  it.j0 = (int)((long long)it.r.steps * split / splits);
  it.j1 = (int)((long long)it.r.steps * (split + 1) / splits);
  const int slot = min(it.s.block, it.s.rows), skip = tall ? wave * kRows : 0;
  it.part = splits > 1 ? m.row0[it.b] + ((int64_t)(block * a.Hkv + it.g) * splits + split) * slot + skip
                       : -1;
  it.tall = tall;
  {
    const int first = block * it.s.block, rows = min(it.s.block, it.s.rows - first);
    it.last_rows = first + (rows - 1) / kRows * kRows;
  }
  it.r0 = min(block * it.s.block + skip, it.s.rows);
  it.r1 = min(it.r0 + kRows, it.s.rows);
  it.own0 = it.j0;
  it.own1 = it.j1;
  if (tall && it.r0 < it.r1) {                 // what these rows see of the block's steps
    const Range own = range_of(a, it.s, it.r0, it.r1);
    it.own1 = min(it.j1, it.r.sinks + own.steps - own.sinks + own.from - it.r.from);
    if (a.sinks == 0) it.own0 = max(it.j0, own.from - it.r.from);
    it.own1 = max(it.own1, it.own0);
  }
  return true;
}

// ---------------------------------------------------------------------------
// operands
// ---------------------------------------------------------------------------

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
  // not live: the loads are issued all the same, all lanes' from one place
  __device__ Pages(const ChunkArgs &a, const int (&id)[2], int g, int lane, bool live = true) {
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
  constexpr int kTogether = 8, K = operands<KV, D>();   // loads in flight together
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

// What the 32 rows of a wavefront see: of the lane's row, of every row, of some row.
struct Sight {
  int lo, hi, all_lo, all_hi, some_lo, some_hi;
};

// Moves the reference above the lane's largest logit (in powers of two). MASKED: what
// weighs nothing against it goes, infinities and NaN too.
template <int D, bool MASKED>
__device__ __forceinline__ void raise_reference(State<D> &st, float top) {
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
// The same for a step's logits (c z: in powers of two, c >= 0).
template <int D, bool MASKED>
__device__ __forceinline__ void move_reference(State<D> &st, const f32x16 &z, float c) {
  float top = max_f(z[0], z[1]);
#pragma unroll
  for (int i = 2; i < 16; ++i) top = max_f(top, z[i]);
  raise_reference<D, MASKED>(st, top * c);
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
    u32x4 p, sees;
    if constexpr (KV != kF32) {
      float x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        // (MASKED: of a page that is not there or that a row does not see, the scale may
        // be anything)
        if constexpr (KV != kFP8) x[i] = w[8 * y + i];
        else if constexpr (MASKED) x[i] = w[8 * y + i] == 0.f ? 0.f : w[8 * y + i] * vs[y];
        else x[i] = w[8 * y + i] * vs[y];
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) p[i] = round_bf16x2(x[2 * i], x[2 * i + 1]);
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
        st.o[db] = mfma(v, p, st.o[db]);
      }
    }
    if (MASKED || KV == kF32) __builtin_amdgcn_sched_barrier(0);
  }
  if constexpr (MASKED)
    if (__any(wild != 0u)) add_classes<KV, D>(st, src, w, seen);
}

// What a wavefront walks: steps j0 .. j1 of its range, in a table row of `pages` pages.
struct Walk {
  const int32_t *table;
  int pages, sinks, shift;   // step j of the range is step j (j < sinks) or j + shift
  int j0, j1;
  __device__ int step(int j) const { return j < sinks ? j : j + shift; }
};

__device__ __forceinline__ bool in_pool(const ChunkArgs &a, int id) {
  return id >= 0 && (int64_t)id < a.num_pages;
}
// One step's by itself.
__device__ __forceinline__ Step step_at(const ChunkArgs &a, const Walk &w, int j) {
  Step x;
#pragma unroll
  for (int pg = 0; pg < 2; ++pg) {
    const int e = 2 * w.step(j) + pg;
    const bool there = j < w.j1 && e < w.pages;
    const int id = w.table[there ? e : 0];
    x.ok[pg] = there && in_pool(a, id);
    x.id[pg] = x.ok[pg] ? id : 0;
  }
  return x;
}
// Page ids of steps j0, j0 + 1, ..: 32 steps' in the lanes of one register, the next 32
// steps' on the way.
struct PageIds {
  int cur, next, k0, lane;
  __device__ static int fetch(const Walk &w, int k, int lane) {
    const int e = 2 * w.step(w.j0 + k + (lane >> 1)) + (lane & 1);
    return w.table[min(e, max(w.pages - 1, 0))];
  }
  __device__ PageIds(const Walk &w, int lane_) : k0(0), lane(lane_) {
    cur = fetch(w, 0, lane);
    next = fetch(w, 32, lane);
  }
  // of step j; j never goes back
  __device__ Step at(const ChunkArgs &a, const Walk &w, int j) {
    const int k = j - w.j0;
    if (k - k0 >= 32) {
      k0 += 32;
      cur = next;
      next = fetch(w, k0 + 32, lane);
    }
    const int s = w.step(j);
    Step x;
#pragma unroll
    for (int pg = 0; pg < 2; ++pg) {
      const int id = __builtin_amdgcn_readlane(cur, 2 * (k - k0) + pg);
      x.ok[pg] = j < w.j1 && 2 * s + pg < w.pages && in_pool(a, id);
      x.id[pg] = x.ok[pg] ? id : 0;
    }
    return x;
  }
};

// Raw logits to powers of two, up to the factor that is returned (not negative:
// the sign of sm_scale is in Q). MASKED: keys that a row does not see to -inf.
template <int KV, bool MASKED>
__device__ __forceinline__ float scale_logits(const ChunkArgs &a, f32x16 &z, uint32_t &seen, int s,
                                              const bool (&ok)[2], const Sight &see,
                                              const float (&ks)[2], int lane) {
  const int hb = lane >> 5;
  seen = 0xffffu;
  if constexpr (KV != kFP8 && !MASKED) return a.scale_log2;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    z[i] *= KV == kFP8 ? a.scale_log2 * ks[i >> 3] : a.scale_log2;
    if constexpr (MASKED) {
      const int pos = (2 * s + (i >> 3)) * kPage + key_of_reg<KV>(i & 7, hb);
      const bool first = pos < a.sinks;
      if (!(ok[i >> 3] && pos < see.hi && (pos >= see.lo || first))) z[i] = -INFINITY;
      if (!(ok[i >> 3] && pos < see.some_hi && (pos >= see.some_lo || first))) seen &= ~(1u << i);
    }
  }
  return 1.f;
}

template <int KV, int D, bool MASKED, class Source>
__device__ __forceinline__ void take_step(State<D> &st, const ChunkArgs &a, const Queries<KV, D> &q,
                                          const Source &src, int s, const bool (&ok)[2],
                                          const Sight &see, const float (&ks)[2],
                                          const float (&vs)[2], int lane) {
  // (the barriers: operands loaded ahead would not fit the registers)
  f32x16 z = logits<KV, D>(src, q);
  __builtin_amdgcn_sched_barrier(0);
  uint32_t seen;
  const float c = scale_logits<KV, MASKED>(a, z, seen, s, ok, see, ks, lane);
  __builtin_amdgcn_sched_barrier(0);
  move_reference<D, MASKED>(st, z, c);
  weigh(st, z, c);
  __builtin_amdgcn_sched_barrier(0);
  add_values<KV, D, MASKED>(st, src, z, seen, vs);
}

template <int KV>
__device__ __forceinline__ void scales_of(const ChunkArgs &a, const int (&id)[2], float (&ks)[2],
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

// Steps [ja, jb) of a walk, which every row sees in full and whose pages are there,
// operands from memory: the next step's K is fetched as soon as this one's has been
// multiplied, and so is V.
template <int KV, int D>
__device__ __forceinline__ void walk_plain(State<D> &st, const ChunkArgs &a, const Walk &w,
                                           const Queries<KV, D> &q, int g, PageIds ids,
                                           const Sight &see, int ja, int jb) {
  const int lane = ids.lane;
  const bool fine[2] = {true, true};
  float ks[2] = {1.f, 1.f}, vs[2] = {1.f, 1.f}, ks1[2] = {1.f, 1.f}, vs1[2] = {1.f, 1.f};
  Held<KV, D> r;
  {
    const Step x = ids.at(a, w, ja);
    const Pages<KV, D> p(a, x.id, g, lane);
    r.load_k(p);
    r.load_v(p);
    scales_of<KV>(a, x.id, ks, vs);
  }
  for (int j = ja;; ++j) {
    const bool more = j + 1 < jb;
    const Step x = ids.at(a, w, j + 1);
    const Pages<KV, D> p(a, x.id, g, lane, more);
    scales_of<KV>(a, x.id, ks1, vs1);
    f32x16 z = logits<KV, D>(r, q);
    __builtin_amdgcn_sched_barrier(0);
    r.load_k(p);
    __builtin_amdgcn_sched_barrier(0);
    uint32_t seen;
    const float c = scale_logits<KV, false>(a, z, seen, 0, fine, see, ks, lane);
    move_reference<D, false>(st, z, c);
    weigh(st, z, c);
    add_values<KV, D, false>(st, r, z, seen, vs);
    __builtin_amdgcn_sched_barrier(0);
    r.load_v(p);
    if (!more) break;
#pragma unroll
    for (int pg = 0; pg < 2; ++pg) {
      ks[pg] = ks1[pg];
      vs[pg] = vs1[pg];
    }
  }
}

// The other steps: those before ja, and those from jb on.
template <int KV, int D>
__device__ __forceinline__ void walk_masked(State<D> &st, const ChunkArgs &a, const Walk &w,
                                            const Queries<KV, D> &q, int g, int lane,
                                            const Sight &see, int ja, int jb) {
  Step x = step_at(a, w, w.j0 < ja ? w.j0 : jb);
  for (int j = w.j0 < ja ? w.j0 : jb; j < w.j1;) {
    const int next = j + 1 == ja ? jb : j + 1;
    const Step x1 = step_at(a, w, next);
    float ks[2] = {1.f, 1.f}, vs[2] = {1.f, 1.f};
    scales_of<KV>(a, x.id, ks, vs);
    take_step<KV, D, true>(st, a, q, Pages<KV, D>(a, x.id, g, lane), w.step(j), x.ok, see, ks, vs, lane);
    x = x1;
    j = next;
  }
}

// ---------------------------------------------------------------------------
// a workgroup's share: its wavefronts' rows over the same steps
// ---------------------------------------------------------------------------

// The pages of two steps (a stage) are brought into LDS as operands, 1 KB each (16 bytes a
// lane, as the lane reads them back; fp8 widened on the way). A wavefront's logits are a
// stage ahead of its weights: while the vector unit weighs one stage's keys, the matrix
// unit multiplies the next one's. So K is staged one ahead of V; there are two buffers of
// either.
// Steps of a stage (256 dims: two would not fit the registers).
template <int D> constexpr int stage_steps() { return D == 256 ? 1 : 2; }
template <int KV, int D> constexpr bool has_lds() { return !q_in_lds<KV, D>(); }
// 16-byte words of a stage's K, and as many of its V.
template <int KV, int D> constexpr int half_words() { return stage_steps<D>() * operands<KV, D>() * 64; }

// A step's K or V operands in LDS, from the lane's first on.
template <int KV, int D>
struct StagedKeys {
  const u32x4 *at;
  __device__ u32x4 key(int c) const { return at[c * 64]; }
};
template <int KV, int D>
struct StagedValues {
  const u32x4 *at;
  __device__ u32x4 value(int y, int db) const { return at[(y * (D / 32) + db) * 64]; }
};

// Operands that a wavefront brings in, on their way: every WAVES-th of a stage's K, and of
// another's V.
template <int KV, int D, int WAVES>
struct Fetch {
  static constexpr int kStage = stage_steps<D>(), kOps = operands<KV, D>(), kEach = kStage * kOps / WAVES;
  static_assert(kOps == v_parts<KV>() * (D / 32) && kStage * kOps % WAVES == 0 &&
                (kOps % WAVES == 0 || WAVES == kStage * kOps), "");
  static constexpr size_t kTile = (size_t)kPage * D * elem_bytes(KV);
  Operand<KV> k[kEach], v[kEach];
  // the step of the wavefront's e-th operand
  __device__ __forceinline__ static int step_of(int e, int wave) {
    if constexpr (WAVES <= kOps) return e * WAVES / kOps;
    else return wave < kOps ? 0 : kStage - 1;
  }
  // ids: the page of step s of the stage, first or second, in lane 4 s + 2 pg
  __device__ __forceinline__ static const char *tile(const ChunkArgs &a, const void *pages, int ids, int s,
                                                     int pg, int g) {
    const int id = __builtin_amdgcn_readlane(ids, 4 * s + 2 * pg);
    return static_cast<const char *>(pages) + ((size_t)id * a.Hkv + g) * kTile;
  }
  __device__ __forceinline__ void issue_k(const ChunkArgs &a, int ids, int g, int wave, int lane) {
    const int i = lane & 31, hb = lane >> 5, tok = key_of_row<KV>(i) & 15;
    const int at = tok * 8 * elem_bytes(KV) + hb * (KV == kF32 ? 16 : 128 * elem_bytes(KV));
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int s = step_of(e, wave), o = (e * WAVES + wave) % kOps;
      uint64_t p0 = reinterpret_cast<uint64_t>(tile(a, a.k_pages, ids, s, 0, g));
      uint64_t p1 = reinterpret_cast<uint64_t>(tile(a, a.k_pages, ids, s, 1, g));
      asm("" : "+s"(p0), "+s"(p1));            // (or the products are the vector unit's, lane by lane)
      // (an address of global memory: a generic one would be waited for with LDS)
      typedef const __attribute__((address_space(1))) decltype(k[e].x) *from;
      k[e].x = *reinterpret_cast<from>((i < 16 ? p0 : p1) + at +
                                       o * (KV == kF32 ? 512 : 256 * elem_bytes(KV)));
    }
  }
  __device__ __forceinline__ void issue_v(const ChunkArgs &a, int ids, int g, int wave, int lane) {
    const int i = lane & 31, hb = lane >> 5;
    const int at = i * 16 * elem_bytes(KV) + hb * (KV == kF32 ? 16 : 8 * elem_bytes(KV));
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int o = (e * WAVES + wave) % kOps, y = o / (D / 32), db = o % (D / 32);
      const char *const base = tile(a, a.v_pages, ids, step_of(e, wave), KV == kF32 ? y >> 1 : y, g) +
                               db * 512 * elem_bytes(KV) + (KV == kF32 ? (y & 1) * 32 : 0);
      v[e] = *reinterpret_cast<const Operand<KV> *>(base + at);
    }
  }
  __device__ __forceinline__ void write_k(u32x4 *to, int wave, int lane) const {
#pragma unroll
    for (int e = 0; e < kEach; ++e) to[(e * WAVES + wave) * 64 + lane] = wide(k[e]);
  }
  __device__ __forceinline__ void write_v(u32x4 *to, int wave, int lane) const {
#pragma unroll
    for (int e = 0; e < kEach; ++e) to[(e * WAVES + wave) * 64 + lane] = wide(v[e]);
  }
};

// A stage's logits as the products gave them.
template <int D> struct Stage {
  f32x16 z[stage_steps<D>()];
  float top[stage_steps<D>()][2];              // the lane's largest of a page's keys
};
template <int D>
__device__ __forceinline__ void find_tops(Stage<D> &p) {
#pragma unroll
  for (int s = 0; s < stage_steps<D>(); ++s)
#pragma unroll
    for (int pg = 0; pg < 2; ++pg) {
      float t = p.z[s][8 * pg];
#pragma unroll
      for (int i = 1; i < 8; ++i) t = max_f(t, p.z[s][8 * pg + i]);
      p.top[s][pg] = t;
    }
}
template <int KV, int D>
__device__ __forceinline__ void multiply_keys(Stage<D> &p, const u32x4 *k, const Queries<KV, D> &q) {
#pragma unroll
  for (int s = 0; s < stage_steps<D>(); ++s)
    p.z[s] = logits<KV, D>(StagedKeys<KV, D>{k + s * operands<KV, D>() * 64}, q);
  find_tops(p);
}

// The stage whose logits are in p, and whose V is at v; K of the next one is at k.
template <int KV, int D>
__device__ __forceinline__ void take_stage(State<D> &st, const ChunkArgs &a, Stage<D> &p, Stage<D> &next,
                                           const Queries<KV, D> &q, const u32x4 *k, const u32x4 *v,
                                           const float (&ks)[stage_steps<D>()][2],
                                           const float (&vs)[stage_steps<D>()][2]) {
  constexpr int kStage = stage_steps<D>();
  float c[kStage][2];                          // factors to powers of two, >= 0
#pragma unroll
  for (int s = 0; s < kStage; ++s)
#pragma unroll
    for (int pg = 0; pg < 2; ++pg) {
      c[s][pg] = KV == kFP8 ? a.scale_log2 * ks[s][pg] : a.scale_log2;
      if constexpr (KV == kFP8) {
        if (c[s][pg] < 0.f) {                  // (a negative scale of a page)
          c[s][pg] = -c[s][pg];
#pragma unroll
          for (int i = 0; i < 8; ++i) p.z[s][8 * pg + i] = -p.z[s][8 * pg + i];
          float t = p.z[s][8 * pg];
#pragma unroll
          for (int i = 1; i < 8; ++i) t = max_f(t, p.z[s][8 * pg + i]);
          p.top[s][pg] = t;
        }
      }
    }
  float top = -INFINITY;
#pragma unroll
  for (int s = 0; s < kStage; ++s) {
    if constexpr (KV == kFP8) top = max_f(top, max_f(p.top[s][0] * c[s][0], p.top[s][1] * c[s][1]));
    else top = max_f(top, max_f(p.top[s][0], p.top[s][1]));
  }
  raise_reference<D, false>(st, KV == kFP8 ? top : top * a.scale_log2);
  // One block of instructions: the products of the next stage's keys, this one's weights and
  // its products with V, operands read from LDS a group ahead of their use. The order is
  // laid out at the end.
  constexpr int kOps = operands<KV, D>(), kDims = D / 32;
#pragma unroll
  for (int s = 0; s < kStage; ++s) {
    next.z[s] = zero16();
#pragma unroll
    for (int o = 0; o < kOps; ++o) {
      const u32x4 x = k[(s * kOps + o) * 64], y = q.at(o);
      if constexpr (KV == kF32) {
#pragma unroll
        for (int e = 0; e < 4; ++e) next.z[s] = mfma(__uint_as_float(x[e]), __uint_as_float(y[e]), next.z[s]);
      } else {
        next.z[s] = mfma(x, y, next.z[s]);
      }
    }
  }
#pragma unroll
  for (int s = 0; s < kStage; ++s) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      p.z[s][i] = exp2_fast(fmaf(p.z[s][i], c[s][i >> 3], -st.ref));
      st.sum += p.z[s][i];
    }
#pragma unroll
    for (int y = 0; y < v_parts<KV>(); ++y) {
      u32x4 w;
      if constexpr (KV != kF32)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float lo = p.z[s][8 * y + 2 * i], hi = p.z[s][8 * y + 2 * i + 1];
          if constexpr (KV == kFP8) {
            lo *= vs[s][y];
            hi *= vs[s][y];
          }
          w[i] = round_bf16x2(lo, hi);
        }
#pragma unroll
      for (int db = 0; db < kDims; ++db) {
        const u32x4 x = v[((s * v_parts<KV>() + y) * kDims + db) * 64];
        if constexpr (KV == kF32) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            st.o[db] = mfma(__uint_as_float(x[e]), p.z[s][4 * y + e], st.o[db]);
        } else {
          st.o[db] = mfma(x, w, st.o[db]);
        }
      }
    }
  }
  find_tops(next);
  {
    constexpr int kGroup = 4, kGroups = 2 * kStage * kOps / kGroup, kPer = KV == kF32 ? 4 : 1;
    constexpr int kVector = KV == kF32 ? 1 : (KV == kFP8 ? 10 : 8) * kStage * 8 / (kGroups * kGroup);
    __builtin_amdgcn_sched_group_barrier(0x100, kGroup, 0);
#pragma unroll
    for (int x = 0; x < kGroups; ++x) {
      if (x + 1 < kGroups) __builtin_amdgcn_sched_group_barrier(0x100, kGroup, 0);
#pragma unroll
      for (int y = 0; y < kGroup * kPer; ++y) {
        __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x2, kVector, 0);
      }
    }
  }
}

// The stages of a workgroup's block from step w.j0 on that start below `end`, whose pages
// are all in the pool. A wavefront takes those that its rows see in full: [ja, jb), whole
// stages from w.j0 on.
//   Page ids and fp8 scales come through vector loads, a stage before they are needed and
// with the data that is waited for anyway: scalar loads would return in any order, among
// the reads of LDS, and a load under a condition would have every stage wait for all.
template <int KV, int D, int WAVES>
__device__ __forceinline__ void walk_staged(State<D> &st, const ChunkArgs &a, const Walk &w,
                                            const Queries<KV, D> &q, int g, int lane, int end, int ja,
                                            int jb, u32x4 *lds, int wave) {
  constexpr int kHalf = half_words<KV, D>(), kStage = stage_steps<D>();
  if (end <= w.j0) return;
  u32x4 *const keys = lds, *const values = lds + 2 * kHalf;
  Fetch<KV, D, WAVES> f;
  // (behind the last step and page: the last's)
  auto pages = [&](int j) {
    const int e = 2 * w.step(min(j + (lane >> 2 & (kStage - 1)), w.j1 - 1)) + (lane >> 1 & 1);
    return w.table[min(e, w.pages - 1)];
  };
  auto scales = [&](int ids) { return KV == kFP8 ? a.kv_scales[2 * (size_t)ids + (lane & 1)] : 1.f; };
  int ids = pages(w.j0), ids1 = pages(w.j0 + kStage), ids2 = pages(w.j0 + 2 * kStage);
  float sc = scales(ids), sc1 = 1.f;           // this stage's, the next one's
  f.issue_k(a, ids, g, wave, lane);
  f.issue_v(a, ids, g, wave, lane);
  f.write_k(keys, wave, lane);
  f.issue_k(a, ids1, g, wave, lane);
  f.write_v(values, wave, lane);
  f.write_k(keys + kHalf, wave, lane);
  __syncthreads();
  Stage<D> p0, p1;
  if (ja == w.j0 && ja < jb) multiply_keys<KV, D>(p0, keys + lane, q);
  __syncthreads();
  // In LDS: this stage's V, the next one's K; on their way: the next one's V, and K of the
  // one after it.
  auto one = [&](int j, int slot, Stage<D> &p, Stage<D> &after) {
    sc1 = scales(ids1);
    const int ids3 = pages(j + 3 * kStage);
    f.issue_v(a, ids1, g, wave, lane);
    f.issue_k(a, ids2, g, wave, lane);
    const u32x4 *const k = keys + (slot ^ 1) * kHalf + lane;
    if (j >= ja && j < jb) {
      float ks[kStage][2], vs[kStage][2];
#pragma unroll
      for (int s = 0; s < kStage; ++s)
#pragma unroll
        for (int pg = 0; pg < 2; ++pg) {
          ks[s][pg] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(sc), 4 * s + 2 * pg));
          vs[s][pg] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(sc), 4 * s + 2 * pg + 1));
        }
      take_stage<KV, D>(st, a, p, after, q, k, values + slot * kHalf + lane, ks, vs);
    } else if (j + kStage == ja && ja < jb) {
      multiply_keys<KV, D>(after, k, q);
    }
    f.write_k(keys + slot * kHalf, wave, lane);
    f.write_v(values + (slot ^ 1) * kHalf, wave, lane);
    ids1 = ids2;
    ids2 = ids3;
    sc = sc1;
    __syncthreads();
  };
  for (int j = w.j0; j < end; j += 2 * kStage) {
    one(j, 0, p0, p1);
    if (j + kStage >= end) break;
    one(j + kStage, 1, p1, p0);
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

// Row r of a sequence's KV head g in q and out.
__device__ __forceinline__ int64_t row_at(const ChunkArgs &a, const Seq &s, int g, int r, int &token) {
  token = div_small(r, a.G);
  return (int64_t)(s.q0 + token) * a.Hq + g * a.G + (r - token * a.G);
}

template <int KV>
__device__ __forceinline__ void store4(const ChunkArgs &a, int64_t at, f32x4 v) {
  if constexpr (KV == kF32)
    *reinterpret_cast<f32x4 *>(static_cast<float *>(a.out) + at) = v;
  else
    *reinterpret_cast<u32x2 *>(static_cast<uint16_t *>(a.out) + at) =
        u32x2{round_bf16x2(v[0], v[1]), round_bf16x2(v[2], v[3])};
}

template <int KV, int D>
__global__ __launch_bounds__(64 * waves_of(KV, D))
__attribute__((amdgpu_waves_per_eu(waves_of(KV, D) / 4)))
void attn_chunk_kernel(ChunkArgs a) {
  constexpr int kWaves = waves_of(KV, D);
  __shared__ __align__(16) u32x4 s_mem[q_in_lds<KV, D>() ? kWaves * operands<KV, D>() * 64
                                                         : 4 * half_words<KV, D>()];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int hb = lane >> 5;
  Item it;
  if (!item_of<kWaves>(a, (int)flat_block(), wave, lane, it)) return;   // (tall: all wavefronts)

  Walk w;
  w.table = a.table + (size_t)it.b * a.stride;
  w.pages = (it.s.len + kPage - 1) / kPage;
  w.sinks = it.r.sinks;
  w.shift = it.r.from - it.r.sinks;
  w.j0 = it.j0;
  w.j1 = it.j1;

  // ---- rows ---------------------------------------------------------------------
  const int r = it.r0 + (lane & 31);
  const bool live = r < it.r1;
  int token;
  const int64_t row = row_at(a, it.s, it.g, live ? r : min(it.r0, it.s.rows - 1), token);
  Sight see;
  see.hi = live ? max(0, it.s.len - it.s.n + token + 1) : 0;
  see.lo = a.window > 0 ? max(0, see.hi - a.window) : 0;
  Queries<KV, D> q;
  {
    constexpr int kBytes = KV == kF32 ? 4 : 2;
    const char *p = static_cast<const char *>(a.q) + row * D * kBytes + hb * 16;
    u32x4 *lds = s_mem + (q_in_lds<KV, D>() ? wave * operands<KV, D>() * 64 + lane : 0);
    q.lds = lds;
#pragma unroll
    for (int c = 0; c < operands<KV, D>(); ++c) {
      u32x4 x = live ? *reinterpret_cast<const u32x4 *>(p + c * 32) : u32x4{0, 0, 0, 0};
      x ^= a.q_sign;
      if constexpr (q_in_lds<KV, D>()) lds[c * 64] = x;   // read by this lane alone
      else q.q[c] = x;
    }
  }
  // Rows that see nothing are walked as if they saw everything, and have no weight
  // afterwards: the other rows' steps stay without masks.
  see.all_hi = see.hi == 0 ? 0x7fffffff : see.hi;
  see.all_lo = see.some_hi = 0;
  see.some_lo = 0x7fffffff;
  if (see.hi > 0) {
    see.all_lo = see.some_lo = see.lo;
    see.some_hi = see.hi;
  }
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) {
    see.all_hi = min(see.all_hi, __shfl_xor(see.all_hi, o, 64));
    see.all_lo = max(see.all_lo, __shfl_xor(see.all_lo, o, 64));
    see.some_hi = max(see.some_hi, __shfl_xor(see.some_hi, o, 64));
    see.some_lo = min(see.some_lo, __shfl_xor(see.some_lo, o, 64));
  }
  see.all_hi = __builtin_amdgcn_readfirstlane(see.all_hi);
  see.all_lo = __builtin_amdgcn_readfirstlane(see.all_lo);
  see.some_hi = __builtin_amdgcn_readfirstlane(see.some_hi);
  see.some_lo = __builtin_amdgcn_readfirstlane(see.some_lo);

  State<D> st;
  auto clear = [&] {
#pragma unroll
    for (int db = 0; db < D / 32; ++db) st.o[db] = zero16();
    st.ref = kNoMax;
    st.sum = 0.f;
  };
  clear();
  if (w.j0 < w.j1) {
    PageIds ids(w, lane);
    // whether all pages are in the pool
    bool fine = true;
    for (int k = 0; w.j0 + k < w.j1; k += 32) {
      const int id = k == 0 ? ids.cur : (k == 32 ? ids.next : PageIds::fetch(w, k, lane));
      const int j = w.j0 + k + (lane >> 1);
      fine &= j >= w.j1 || 2 * w.step(j) + (lane & 1) >= w.pages || in_pool(a, id);
    }
    fine = !__any(!fine);
    // steps that every row sees in full
    int ja = max(it.own0, (see.all_lo + kKeys - 1) / kKeys - w.shift);
    int jb = max(ja, min(it.own1, see.all_hi / kKeys - w.shift));
    if (ja < w.sinks) ja = min(jb, w.sinks);
    if (see.some_hi == 0) it.own1 = it.own0;   // (no row sees anything)
    if (!fine || !has_plain<KV, D>() || it.own0 >= it.own1) ja = jb = it.own0;
    bool staged = false;
    if constexpr (has_lds<KV, D>()) {
      if (it.tall && fine) {
        // whole stages; those that start beyond what the block's last 32 rows all see are
        // nobody's
        constexpr int kStage = stage_steps<D>();
        ja = w.j0 + (ja - w.j0 + kStage - 1) / kStage * kStage;
        jb = max(ja, w.j0 + (jb - w.j0) / kStage * kStage);
        const int last = div_small(it.last_rows, a.G);
        const int end = min(w.j1, max(0, it.s.len - it.s.n + last + 1) / kKeys - w.shift);
        walk_staged<KV, D, kWaves>(st, a, w, q, it.g, opaque(lane), end, ja, jb, s_mem, wave);
        staged = true;
        if (ja >= jb) ja = jb = it.own0;
      }
    }
    // A product gives 0 * inf = NaN where a weight is zero. Rather than test V on the way, a
    // wavefront whose result is not finite walks its steps again with masks, which keep
    // infinities and NaN of V out of the products. (Not for rows that see nothing, nor for
    // those that a NaN logit has made NaN.)
    w.j0 = it.own0;
    w.j1 = it.own1;
    for (;;) {
      if (has_plain<KV, D>() && !staged && ja < jb)
        walk_plain<KV, D>(st, a, w, q, it.g, PageIds(w, opaque(lane)), see, ja, jb);
      if (w.j0 < w.j1) walk_masked<KV, D>(st, a, w, q, it.g, opaque(lane), see, ja, jb);
      staged = false;
      st.sum += other_half(st.sum);
      if (ja >= jb) break;
      float top = 0.f;
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) top = max_f(top, __builtin_fabsf(st.o[db][i]));
      if (!__any(!(top < INFINITY) && see.hi > 0 && st.sum == st.sum)) break;
      ja = jb = w.j0;
      clear();
    }
  }
  if (see.hi == 0) st.sum = 0.f;
  if (!live) return;
  const float inv = st.sum == 0.f ? 0.f : 1.f / st.sum;
  const float lse = st.sum == 0.f ? -INFINITY : st.ref + log2f(st.sum);
  const int64_t part = it.part + (lane & 31);
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int y = 0; y < 4; ++y) {
      f32x4 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = st.sum == 0.f ? 0.f : st.o[db][4 * y + e] * inv;
      const int d = 32 * db + 8 * y + 4 * hb;
      if (it.part >= 0) *reinterpret_cast<f32x4 *>(a.part_o + part * D + d) = v;
      else store4<KV>(a, row * D + d, v);
    }
  if (hb == 0) {
    if (it.part >= 0) a.part_lse[part] = lse;
    else if (a.lse) a.lse[row] = lse * kLn2;
  }
}

// ---------------------------------------------------------------------------
// merge: the rows of a block over its splits
// ---------------------------------------------------------------------------

constexpr int kMergeThreads = 256;

template <int KV, int D>
__global__ __launch_bounds__(kMergeThreads) void merge_chunk_kernel(ChunkArgs a) {
  const MapOf m = map_of(a);
  const int lane = threadIdx.x & 63, total = m.head[kMapMerge];
  for (int w = blockIdx.x; w < total; w += gridDim.x) {
    const int b = find(m.merge, a.batch, w, lane);
    const Seq s = seq_of(a, b, kRows * waves_of(KV, D));
    const int off = w - m.merge[b], block = div_small(off, a.Hkv), g = off - block * a.Hkv;
    const int splits = m.splits[b], slot = min(s.block, s.rows);
    if (off < 0 || block >= s.blocks || splits < 2) continue;   // (offsets that do not ascend)
    const int64_t row0 = m.row0[b] + (int64_t)off * splits * slot;
    const int r0 = block * s.block, rows = min(s.rows - r0, s.block);
    for (int i = threadIdx.x; i < rows * (D / 4); i += kMergeThreads) {
      const int rl = i / (D / 4), d = i % (D / 4) * 4;
      float mx = -INFINITY, l = 0.f;
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
      for (int t = 0; t < splits; ++t) {
        const int64_t at = row0 + (int64_t)t * slot + rl;
        const float lse = a.part_lse[at];
        if (lse == -INFINITY) continue;          // no key seen
        const f32x4 v = *reinterpret_cast<const f32x4 *>(a.part_o + at * D + d);
        const float mm = max_f(mx, lse);
        const float f = exp2_fast(mx - mm), x = exp2_fast(lse - mm);
        mx = mm;
        l = l * f + x;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = (f == 0.f ? 0.f : o[e] * f) + (x == 0.f ? 0.f : v[e] * x);
      }
      int token;
      const int64_t row = row_at(a, s, g, r0 + rl, token);
      f32x4 res;
#pragma unroll
      for (int e = 0; e < 4; ++e) res[e] = l == 0.f ? 0.f : o[e] / l;
      store4<KV>(a, row * D + d, res);
      if (d == 0 && a.lse) a.lse[row] = l == 0.f ? -INFINITY : (mx + log2f(l)) * kLn2;
    }
  }
}

template <int KV, int D>
void launch_d(const ChunkArgs &a, hipStream_t s) {
  constexpr int kWaves = waves_of(KV, D);
  const dim3 grid((unsigned)std::min<long long>(a.grid, kAlongX), 1, (unsigned)((a.grid + kAlongX - 1) / kAlongX));
  hipLaunchKernelGGL(chunk_plan_kernel<kWaves>, dim3(1), dim3(kScanThreads), 0, s, a);
  hipLaunchKernelGGL((attn_chunk_kernel<KV, D>), grid, dim3(64 * kWaves), 0, s, a);
  if (a.part_rows > 0)
    hipLaunchKernelGGL((merge_chunk_kernel<KV, D>), dim3(4 * a.target), dim3(kMergeThreads), 0, s, a);
}

template <int KV>
void launch_kv(const ChunkArgs &a, hipStream_t s) {
  if (a.D == 64) launch_d<KV, 64>(a, s);
  else if (a.D == 128) launch_d<KV, 128>(a, s);
  else launch_d<KV, 256>(a, s);
}

}  // namespace

hipError_t launch_attn_chunk(const ChunkArgs &a, hipStream_t s) {
  if (a.kv_type == kF32) launch_kv<kF32>(a, s);
  else if (a.kv_type == kBF16) launch_kv<kBF16>(a, s);
  else launch_kv<kFP8>(a, s);
  return hipGetLastError();
}

}  // namespace kap

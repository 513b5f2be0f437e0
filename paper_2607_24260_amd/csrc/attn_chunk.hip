// Attention of ragged chunks of new tokens -- from one token a sequence to whole
// prompts -- over the paged cache, causal, with a sliding window and sinks or without.
//
// The rows of a (sequence, KV head) are its new tokens times the query heads of the
// KV head, token by token. A wavefront holds 32 rows and walks 32 keys (two pages) a
// step (attn_tiles.h): S^T = K Q^T, o <- o e^(m - m') + V^T e^(S^T - m'), with a running
// reference m that moves only when a logit exceeds it. Rows see positions lo <= t < hi and
// t < sinks; a block of rows walks the steps that hold its sinks, then those from its
// lowest lo to its highest hi, those that every row sees in full without masks.
//
// A step reads 2 * 32 * D elements and multiplies 4 * 32 * 32 * D for 32 rows: with few
// rows memory bounds it, with many the matrix units. So single tokens and short chunks are
// taken 32 rows at a time, a workgroup's wavefronts sharing the keys ("team"); chunks of
// more than 128 rows by up to 256 rows over the same keys, staged through LDS once for all
// ("tall": a wavefront reads 1/8 of what it multiplies); and short sequences by the
// hundred by a wavefront each, which meets no other ("solo": 1000 of 300 tokens 270 us,
// by teams 465). One launch does all kinds at once. On one device, bf16, 32 heads over 8
// KV heads of 128 dims:
//   one token at 2048: 14.5 us; 64 tokens that see 4096 of 32768: 200 us, 5.4 TB/s;
//   8192-token prompt: 560 us, 0.98 PFLOP/s (fp8: two chunks of 2048 at 32768: 1000 us,
//   0.90); 4096 tokens at 16384: 1.1 PFLOP/s. The same loop without the fetches runs at 1.2,
//   also without exponentials and sums at 1.25, also without LDS reads at 1.4: eight
//   wavefronts' operands, 1 KB for every product of 32 cycles, take all that LDS gives
//   (128 bytes a cycle), so the products of the four matrix units and the reads of the one
//   LDS each last as long as the other; the matrix units are busy half of the time.
#include "attn_tiles.h"
#include "block_scan.h"
#include "chunk_cut.h"

#include <algorithm>
#include <type_traits>

namespace kap {
namespace {

constexpr int waves_of(int kv, int D) { return chunk_waves(kv, D); }

// ---------------------------------------------------------------------------
// work map
// ---------------------------------------------------------------------------

// Sum over a wavefront, the same in every lane: a float by row shifts (no LDS), a whole
// number exactly.
__device__ __forceinline__ float wave_total(float x) {
  auto from = [](float v, auto shift, auto rows) {
    return __int_as_float(dpp_or_zero<decltype(shift)::value, decltype(rows)::value>(__float_as_int(v)));
  };
  using std::integral_constant;
  x += from(x, integral_constant<int, 0x111>(), integral_constant<int, 0xF>());
  x += from(x, integral_constant<int, 0x112>(), integral_constant<int, 0xF>());
  x += from(x, integral_constant<int, 0x114>(), integral_constant<int, 0xF>());
  x += from(x, integral_constant<int, 0x118>(), integral_constant<int, 0xF>());
  x += from(x, integral_constant<int, 0x142>(), integral_constant<int, 0xA>());
  x += from(x, integral_constant<int, 0x143>(), integral_constant<int, 0xC>());
  return __int_as_float(lane63(__float_as_int(x)));
}
__device__ __forceinline__ long long wave_total(long long x) {
  return __shfl(wave_incl(x, threadIdx.x & 63), 63, 64);
}
__device__ __forceinline__ long long wave_total(int x) {   // x >= 0
  return ((long long)lane63(wave_scan_add(x >> 16)) << 16) + lane63(wave_scan_add(x & 0xffff));
}

// What a workgroup does, or with solo blocks a wavefront.
struct Part {
  Seq s;
  int b;
  Kind kind;
  int splits, off;             // off: of the parts of a sequence
  int64_t row0;                // rows of the partials of a sequence, from here on
  int ticket;                  // arrival counters of a sequence, from here on
};
// Parts are handed out the longest first (one that starts late would end alone): sequences
// in classes of a quarter of an octave of their parts' steps.
constexpr int kClasses = 8;
__device__ __forceinline__ int class_of(float longest, float steps) {
  return (int)fminf(fmaxf(4.f * __builtin_amdgcn_logf(longest / fmaxf(steps, 1e-3f)), 0.f),
                    (float)(kClasses - 1));
}

// The map of a call with more blocks than run at once, or more sequences than lanes, is made
// once, by a launch before (6 to 8 us, 26 of more than 64 sequences; a workgroup that makes
// it for itself: 2 to 3): the parts of each kind; sequences in the order of their classes;
// for each of them, in that order, the parts of each kind before it, and what is its own.
struct MapSeq {
  int b, splits, ticket, q0;
  int64_t row0;
  int n, len;
};
struct MapOf {
  MapSeq *seq;
  int32_t *head, *first, *order;   // first: [3][batch]
};
__device__ __forceinline__ MapOf map_of(const ChunkArgs &a) {
  MapOf m;
  m.seq = reinterpret_cast<MapSeq *>(a.map);
  m.head = reinterpret_cast<int32_t *>(m.seq + a.batch);
  m.first = m.head + 4;
  m.order = m.first + 3 * (size_t)a.batch;
  return m;
}

// Of up to 64 sequences, by one wavefront.
template <int WAVES>
__global__ __launch_bounds__(64) void chunk_plan_small_kernel(ChunkArgs a) {
  const MapOf m = map_of(a);
  const int lane = threadIdx.x;
  Seq s{};
  Info f{};
  if (lane < a.batch) {
    s = seq_of(a, lane);
    f = info_of<WAVES>(a, s);
  }
  auto sum = [&](auto g) { return wave_total(g(f)); };
  auto most = [&](float x) { return __int_as_float(lane63(wave_scan_max(__float_as_int(x)))); };
  const Cut c = cut_of<WAVES, true>(a, sum, [&](auto g) { return most(g(f)); });
  const Kind kind = c.kind(a, f);
  const Parts x = parts_of<WAVES>(a, c, f);
  const float steps = part_steps(c, kind, f);
  const int cls = class_of(most(steps), steps);
  const int merged = wave_scan_add(x.merges) - x.merges;
  const long long rows = wave_incl(x.rows, lane) - x.rows;
  int at = 0, before[3] = {0, 0, 0}, first[3] = {0, 0, 0}, place = 0;
#pragma unroll 1
  for (int i = 0; i < kClasses; ++i) {
    const bool in = lane < a.batch && cls == i;
    const unsigned long long here = __ballot(in);
    if (!here) continue;
    if (in) place = at + __popcll(here & ((1ull << lane) - 1));
    at += __popcll(here);
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      const int n = in && kind == k ? x.parts : 0, incl = wave_scan_add(n);
      if (in) first[k] = before[k] + incl - n;
      before[k] += lane63(incl);
    }
  }
  if (lane < a.batch) {
#pragma unroll
    for (int k = 0; k < 3; ++k) m.first[k * a.batch + place] = first[k];
    m.seq[place] = MapSeq{lane, x.splits, merged, s.q0, rows, s.n, s.len};
  }
  if (lane == 0)
    for (int k = 0; k < 3; ++k) m.head[k] = before[k];
}

// Of more, by a workgroup.
template <int WAVES>
__global__ __launch_bounds__(kScanThreads) void chunk_plan_kernel(ChunkArgs a) {
  __shared__ long long s_scan[5][kScanWaves];
  __shared__ double s_sum[kScanWaves];
  __shared__ int s_count[kClasses][kScanWaves];
  const MapOf m = map_of(a);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  // (the first sequence of each thread, kept: often there are no others)
  auto info_at = [&](int b) { return b < a.batch ? info_of<WAVES>(a, seq_of(a, b)) : Info{}; };
  const Info kept = info_at(threadIdx.x);
  // f of all sequences, folded by `in_wave` over each wavefront and by `fold` over those
  auto over_all = [&](auto f, auto in_wave, auto fold) {
    typedef decltype(in_wave(f(Info{}))) T;
    T x = in_wave(f(kept));
    for (int b0 = kScanThreads; b0 < a.batch; b0 += kScanThreads)
      x = fold(x, in_wave(f(info_at(b0 + threadIdx.x))));
    __syncthreads();
    if (lane == 0) s_sum[wave] = (double)x;
    __syncthreads();
    return in_wave(lane < kScanWaves ? (T)s_sum[lane] : (T)0);
  };
  auto sum = [&](auto f) {
    return over_all(f, [](auto x) { return wave_total(x); }, [](auto x, auto y) { return x + y; });
  };
  auto greatest = [&](auto f) {
    return over_all(
        f, [](float x) { return __int_as_float(lane63(wave_scan_max(__float_as_int(x)))); },
        [](float x, float y) { return fmaxf(x, y); });
  };
  const Cut c = cut_of<WAVES, true>(a, sum, greatest);
  const float longest = greatest([&](const Info &f) { return part_steps(c, c.kind(a, f), f); });
  // their order: how many there are of each class, then the place of each
  int count[kClasses];
#pragma unroll
  for (int i = 0; i < kClasses; ++i) count[i] = 0;
  for (int pass = 0; pass < 2; ++pass) {
    for (int b0 = 0; b0 < a.batch; b0 += kScanThreads) {
      const int b = b0 + threadIdx.x;
      int cls = -1;
      if (b < a.batch) {
        const Info f = b0 == 0 ? kept : info_at(b);
        cls = class_of(longest, part_steps(c, c.kind(a, f), f));
      }
      int rank = 0;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kClasses; ++i) {
        const unsigned long long here = __ballot(cls == i);
        if (cls == i) rank = __popcll(here & ((1ull << lane) - 1));
        if (lane == 0) s_count[i][wave] = __popcll(here);
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kClasses; ++i) {
        const int mine = lane < kScanWaves ? s_count[i][lane] : 0, incl = wave_scan_add(mine);
        const int all = lane63(incl);
        const int before =
            __builtin_amdgcn_readlane(incl - mine, __builtin_amdgcn_readfirstlane(wave));
        if (pass == 1 && cls == i) m.order[count[i] + before + rank] = b;
        count[i] += all;
      }
    }
    if (pass == 0) {                           // of the classes before
      int run = 0;
#pragma unroll
      for (int i = 0; i < kClasses; ++i) {
        const int n = count[i];
        count[i] = run;
        run += n;
      }
    }
  }
  __syncthreads();
  long long before[5] = {0, 0, 0, 0, 0};       // parts of each kind, merges, rows
  for (int i0 = 0; i0 < a.batch; i0 += kScanThreads) {
    const int i = i0 + threadIdx.x;
    const bool in = i < a.batch;
    Kind k = kTeam;
    Parts p{0, 0, 0, 0};
    Seq s{};
    int b = 0;
    if (in) {
      b = m.order[i];
      s = seq_of(a, b);
      const Info f = info_of<WAVES>(a, s);
      k = c.kind(a, f);
      p = parts_of<WAVES>(a, c, f);
    }
    const long long x[5] = {k == kTall ? p.parts : 0, k == kTeam ? p.parts : 0, k == kSolo ? p.parts : 0,
                            p.merges, p.rows};
    long long incl[5], total[5];
    scan(x, incl, total, s_scan);
    if (in) {
#pragma unroll
      for (int k = 0; k < 3; ++k) m.first[k * (size_t)a.batch + i] = (int)(before[k] + incl[k] - x[k]);
      m.seq[i] = MapSeq{b,   p.splits, (int)(before[3] + incl[3] - x[3]), s.q0, before[4] + incl[4] - x[4],
                        s.n, s.len};
    }
#pragma unroll
    for (int k = 0; k < 5; ++k) before[k] += total[k];
  }
  if (threadIdx.x == 0)
    for (int k = 0; k < 3; ++k) m.head[k] = (int)before[k];
}

// The last of n ascending sums that is at most w (by a whole wavefront); value: the lane's
// of the first 64.
__device__ __forceinline__ int find(const int32_t *first, int value, int n, int w, int lane) {
  if (n <= 64)
    return __builtin_amdgcn_readfirstlane(__popcll(__ballot(lane < n && value <= w)) - 1);
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int step = (hi - lo + 63) / 64, i = lo + lane * step;
    const unsigned long long hit = __ballot(i < hi && first[min(i, hi - 1)] <= w);
    lo += (__popcll(hit) - 1) * step;
    hi = min(lo + step, hi);
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

template <int WAVES>
__device__ __forceinline__ bool part_of(const ChunkArgs &a, int w, int wave, int lane, Part &p) {
  if (a.map) {
    const MapOf m = map_of(a);
    const int head[3] = {m.head[0], m.head[1], m.head[2]};
    int value[3];
#pragma unroll
    for (int k = 0; k < 3; ++k) value[k] = m.first[k * (size_t)a.batch + min(lane, a.batch - 1)];
    const int k = place(head[0], head[1], WAVES, wave, w);
    if (w >= pick(k == 0, head[0], pick(k == 1, head[1], head[2]))) return false;
    const int32_t *first = m.first + k * (size_t)a.batch;
    const int i = find(first, pick(k == 0, value[0], pick(k == 1, value[1], value[2])), a.batch, w, lane);
    if (i < 0) return false;
    const MapSeq x = m.seq[i];
    p.s = Seq{x.q0, x.n, x.len, x.n * a.G};
    p.b = x.b;
    p.kind = (Kind)k;
    p.splits = x.splits;
    p.off = w - first[i];
    p.row0 = x.row0;
    p.ticket = x.ticket;
    return p.splits > 0 && p.off >= 0;         // (offsets that do not ascend)
  }
  Seq s{};
  Info f{};
  if (lane < a.batch) {
    s = seq_of(a, lane);
    f = info_of<WAVES>(a, s);
  }
  const Cut c = cut_of<WAVES, false>(a, [&](auto g) { return wave_total(g(f)); }, 0);
  const Kind kind = c.kind(a, f);
  const Parts x = parts_of<WAVES>(a, c, f);
  const int k = place(lane63(wave_scan_add(kind == kTall ? x.parts : 0)),
                      lane63(wave_scan_add(kind == kTeam ? x.parts : 0)), WAVES, wave, w);
  const int n = kind == k ? x.parts : 0, incl = wave_scan_add(n);
  const unsigned long long hit = __ballot(w >= incl - n && w < incl);
  if (!hit) return false;
  const int l = __builtin_amdgcn_readfirstlane(__ffsll((long long)hit) - 1);
  auto of = [&](int v) { return __builtin_amdgcn_readlane(v, l); };
  p.s = Seq{of(s.q0), of(s.n), of(s.len), of(s.rows)};
  p.b = l;
  p.kind = (Kind)k;
  p.splits = of(x.splits);
  p.off = w - of(incl - n);
  p.row0 = 0;
  p.ticket = 0;
  if (p.splits > 1) {
    const int merged = wave_scan_add(x.merges) - x.merges;
    const long long rows = wave_incl(x.rows, lane) - x.rows;
    p.ticket = of(merged);
    p.row0 = (int64_t)of((int)(rows >> 32)) << 32 | (uint32_t)of((int)rows);
  }
  return true;
}

// What a wavefront does: rows [r0, r1) of a sequence's KV head g over steps of its block's
// range.
struct Item {
  Seq s;
  int b, g, r0, r1;
  Kind kind;
  Range r;
  int j0, j1;        // the workgroup's (tall) or wavefront's steps
  int own0, own1;    // of which these rows see something in [own0, own1)
  int last_rows;     // tall: where the block's last wavefront with rows starts
};
// Where its results go.
struct Goal {
  int64_t first_part, part;   // the block's partials, this part's
  int splits, ticket;
  Kind kind;
  int q0, rows, g;   // of the sequence; KV head
  int base, height;  // the block's first row, its rows
};

template <int WAVES>
__device__ __forceinline__ bool item_of(const ChunkArgs &a, int w, int wave, int lane, Item &it,
                                        Goal &goal) {
  Part p;
  if (!part_of<WAVES>(a, w, wave, lane, p)) return false;
  it.b = p.b;
  it.kind = p.kind;
  it.s = p.s;
  const int size = p.kind == kTall ? kRows * WAVES : kRows, blocks = (it.s.rows + size - 1) / size;
  int block, split = 0;
  if (p.kind == kTall) {                       // the longest first; KV heads share out the XCDs
    const int at = div_small(p.off, a.Hkv);
    it.g = p.off - at * a.Hkv;
    block = div_small(at, p.splits);
    split = at - block * p.splits;
    block = blocks - 1 - block;
  } else {
    const int at = div_small(p.off, p.splits);
    split = p.off - at * p.splits;
    block = div_small(at, a.Hkv);
    it.g = at - block * a.Hkv;
  }
  if (block < 0 || block >= blocks) return false;   // (offsets that do not ascend)
  const int base = block * size, height = min(size, it.s.rows - base);
  it.r = range_of(a, it.s, base, base + height);
  it.j0 = (int)((long long)it.r.steps * split / p.splits);
  it.j1 = (int)((long long)it.r.steps * (split + 1) / p.splits);
  const int slot = min(size, it.s.rows), at = block * a.Hkv + it.g;
  goal.first_part = p.row0 + (int64_t)at * p.splits * slot;
  goal.part = goal.first_part + (int64_t)split * slot;
  goal.splits = p.splits;
  goal.ticket = p.ticket + at;
  goal.kind = p.kind;
  goal.q0 = it.s.q0;
  goal.rows = it.s.rows;
  goal.g = it.g;
  goal.base = base;
  goal.height = height;
  const int skip = p.kind == kTall ? wave * kRows : 0;
  it.r0 = min(base + skip, it.s.rows);
  it.r1 = min(it.r0 + kRows, base + height);
  it.last_rows = base + (height - 1) / kRows * kRows;
  if (p.kind == kTeam) {
    const int n = it.j1 - it.j0;
    it.j1 = it.j0 + (int)((long long)n * (wave + 1) / WAVES);
    it.j0 += (int)((long long)n * wave / WAVES);
  }
  it.own0 = it.j0;
  it.own1 = it.j1;
  if (p.kind == kTall && it.r0 < it.r1) {      // what these rows see of the block's steps
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

// The tiles of a KV head: page id's begin id * stride bytes from these.
struct Tiles {
  const char *k, *v;
  uint32_t stride;
  __device__ const char *key(int id) const { return k + (uint64_t)(uint32_t)id * stride; }
  __device__ const char *value(int id) const { return v + (uint64_t)(uint32_t)id * stride; }
};

// Operands of a step in memory, for the lane that multiplies them.
template <int KV, int D>
struct Pages {
  const char *k, *v[2];
  // not live: the loads are issued all the same, all lanes' from one place
  __device__ Pages(const Tiles &head, const int (&id)[2], int lane, bool live = true) {
    const int i = lane & 31, hb = lane >> 5, tok = key_of_row<KV>(i) & 15;
    const int k_at = tok * 8 * elem_bytes(KV) + hb * (KV == kF32 ? 16 : 128 * elem_bytes(KV));
    const int v_at = i * 16 * elem_bytes(KV) + hb * (KV == kF32 ? 16 : 8 * elem_bytes(KV));
    k = head.key(i < 16 && live ? id[0] : id[1]) + (live ? k_at : 0);
#pragma unroll
    for (int pg = 0; pg < 2; ++pg) v[pg] = head.value(id[pg]) + (live ? v_at : 0);
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
//   Weights meet 16-bit V as two parts of bf16, what the first rounds off in the second (2^-16
// of a weight is left), for an error against 64 bits of 0.0017 instead of 0.0023, which is what
// rounding the result costs. Memory bounds most walks that come here, which hardly notice the
// second products (one token at 2048 14.2 to 14.5 us, 64 with a window of 4096 199 to 200; 64
// chunks of 12 tokens at 4000 224 to 227); blocks that share their keys in the caches do (fp8:
// 64 of 24 tokens at 4000 225 to 248 us).
template <int KV, int D, bool MASKED, class Source>
__device__ __forceinline__ void add_values(State<D> &st, const Source &src, const f32x16 &w,
                                           uint32_t seen, const float (&vs)[2]) {
  uint32_t wild = 0;
#pragma unroll
  for (int y = 0; y < v_parts<KV>(); ++y) {
    u32x4 p, rest, sees;
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
      for (int i = 0; i < 4; ++i) {
        p[i] = round_bf16x2(x[2 * i], x[2 * i + 1]);
        rest[i] = round_bf16x2(x[2 * i] - __uint_as_float(p[i] << 16),
                               x[2 * i + 1] - __uint_as_float(p[i] & 0xffff0000u));
        // (infinite weights, of pages of such a scale, leave nothing)
        if constexpr (KV == kFP8) rest[i] &= __builtin_fabsf(vs[y]) < INFINITY ? ~0u : 0u;
      }
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
        st.o[db] = mfma(v, rest, st.o[db]);
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
// multiplied, and so is V. Page ids and scales come through vector loads a step before they
// are needed: in order with the others, so that none is waited for by itself.
template <int KV, int D>
__device__ __forceinline__ void walk_plain(State<D> &st, const ChunkArgs &a, const Walk &w,
                                           const Queries<KV, D> &q, const Tiles &head, int lane,
                                           const Sight &see, int ja, int jb) {
  // lanes 4 i + 2 pg (+ 1): of page pg
  auto pages = [&](int j) { return w.table[2 * w.step(min(j, jb - 1)) + (lane >> 1 & 1)]; };
  auto scales = [&](int ids) { return KV == kFP8 ? a.kv_scales[2 * (size_t)ids + (lane & 1)] : 1.f; };
  const bool fine[2] = {true, true};
  int ids = pages(ja), ids1 = pages(ja + 1);
  float sc = scales(ids);
  Held<KV, D> r;
  {
    const int id[2] = {__builtin_amdgcn_readlane(ids, 0), __builtin_amdgcn_readlane(ids, 2)};
    const Pages<KV, D> p(head, id, lane);
    r.load_k(p);
    r.load_v(p);
  }
  for (int j = ja;; ++j) {
    const bool more = j + 1 < jb;
    const int id[2] = {__builtin_amdgcn_readlane(ids1, 0), __builtin_amdgcn_readlane(ids1, 2)};
    const Pages<KV, D> p(head, id, lane, more);
    const float sc1 = scales(ids1);
    ids1 = pages(j + 2);
    float ks[2] = {1.f, 1.f}, vs[2] = {1.f, 1.f};
    if constexpr (KV == kFP8)
#pragma unroll
      for (int pg = 0; pg < 2; ++pg) {
        ks[pg] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(sc), 2 * pg));
        vs[pg] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(sc), 2 * pg + 1));
      }
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
    sc = sc1;
  }
}

// The other steps: those before ja, and those from jb on.
template <int KV, int D>
__device__ __forceinline__ void walk_masked(State<D> &st, const ChunkArgs &a, const Walk &w,
                                            const Queries<KV, D> &q, const Tiles &head, int lane,
                                            const Sight &see, int ja, int jb) {
  Step x = step_at(a, w, w.j0 < ja ? w.j0 : jb);
  for (int j = w.j0 < ja ? w.j0 : jb; j < w.j1;) {
    const int next = j + 1 == ja ? jb : j + 1;
    const Step x1 = step_at(a, w, next);
    float ks[2] = {1.f, 1.f}, vs[2] = {1.f, 1.f};
    scales_of<KV>(a, x.id, ks, vs);
    take_step<KV, D, true>(st, a, q, Pages<KV, D>(head, x.id, lane), w.step(j), x.ok, see, ks, vs, lane);
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
// either. (8192-token prompt: 590 us, 639 with every wavefront reading the pages by itself;
// 549 with page ids and scales a stage ahead. Loads straight into LDS, with no registers on
// the way, were no faster: 0.985 against 1.0 PFLOP/s at 4096 tokens on 16384.)
// Steps of a stage (256 dims: two would not fit the registers).
template <int D> constexpr int stage_steps() { return D == 256 ? 1 : 2; }
template <int KV, int D> constexpr bool has_lds() { return !q_in_lds<KV, D>(); }
// 16-byte words of a stage's K, and as many of its V.
template <int KV, int D> constexpr int half_words() { return stage_steps<D>() * operands<KV, D>() * 64; }

// A step's K operands in LDS, from the lane's first on.
template <int KV, int D>
struct StagedKeys {
  const u32x4 *at;
  __device__ u32x4 key(int c) const { return at[c * 64]; }
};

// Operands that a wavefront brings in, on their way: every WAVES-th of a stage's K, and of
// another's V.
template <int KV, int D, int WAVES>
struct Fetch {
  static constexpr int kStage = stage_steps<D>(), kOps = operands<KV, D>(), kEach = kStage * kOps / WAVES;
  static_assert(kOps == v_parts<KV>() * (D / 32) && kStage * kOps % WAVES == 0 &&
                (kOps % WAVES == 0 || WAVES == kStage * kOps), "");
  Operand<KV> k[kEach], v[kEach];
  // the step of the wavefront's e-th operand
  __device__ __forceinline__ static int step_of(int e, int wave) {
    if constexpr (WAVES <= kOps) return e * WAVES / kOps;
    else return wave < kOps ? 0 : kStage - 1;
  }
  // ids: the page of step s of the stage, first or second, in lane 4 s + 2 pg
  __device__ __forceinline__ static int page(int ids, int s, int pg) {
    return __builtin_amdgcn_readlane(ids, 4 * s + 2 * pg);
  }
  __device__ __forceinline__ void issue_k(const Tiles &head, int ids, int wave, int lane) {
    const int i = lane & 31, hb = lane >> 5, tok = key_of_row<KV>(i) & 15;
    const int at = tok * 8 * elem_bytes(KV) + hb * (KV == kF32 ? 16 : 128 * elem_bytes(KV));
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int s = step_of(e, wave), o = (e * WAVES + wave) % kOps;
      uint64_t p0 = reinterpret_cast<uint64_t>(head.key(page(ids, s, 0)));
      uint64_t p1 = reinterpret_cast<uint64_t>(head.key(page(ids, s, 1)));
      asm("" : "+s"(p0), "+s"(p1));            // (or the products are the vector unit's, lane by lane)
      // (an address of global memory: a generic one would be waited for with LDS)
      typedef const __attribute__((address_space(1))) decltype(k[e].x) *from;
      k[e].x = *reinterpret_cast<from>((i < 16 ? p0 : p1) + at +
                                       o * (KV == kF32 ? 512 : 256 * elem_bytes(KV)));
    }
  }
  __device__ __forceinline__ void issue_v(const Tiles &head, int ids, int wave, int lane) {
    const int i = lane & 31, hb = lane >> 5;
    const int at = i * 16 * elem_bytes(KV) + hb * (KV == kF32 ? 16 : 8 * elem_bytes(KV));
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int o = (e * WAVES + wave) % kOps, y = o / (D / 32), db = o % (D / 32);
      const char *const base = head.value(page(ids, step_of(e, wave), KV == kF32 ? y >> 1 : y)) +
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
//   Weights meet 16-bit V rounded to bf16 once (off by 2^-8 of each at most): the matrix units
// bound this loop, and a second part's products took an 8192-token prompt from 550 to 747 us
// (fp8, 2 x 2048 tokens at 32768: 995 to 1347), for errors against 64 bits of 0.0016 instead of
// 0.0021 (0.0017, 0.0023), of which rounding the result is 0.0016.
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
                                            const Queries<KV, D> &q, const Tiles &head, int lane, int end, int ja,
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
  f.issue_k(head, ids, wave, lane);
  f.issue_v(head, ids, wave, lane);
  f.write_k(keys, wave, lane);
  f.issue_k(head, ids1, wave, lane);
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
    f.issue_v(head, ids1, wave, lane);
    f.issue_k(head, ids2, wave, lane);
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
__device__ __forceinline__ int64_t row_at(const ChunkArgs &a, int q0, int g, int r, int &token) {
  token = token_of(a, r);
  return (int64_t)(q0 + token) * a.Hq + g * a.G + (r - token * a.G);
}

template <int KV>
__device__ __forceinline__ void store4(const ChunkArgs &a, int64_t at, f32x4 v) {
  if constexpr (KV == kF32)
    *reinterpret_cast<f32x4 *>(static_cast<float *>(a.out) + at) = v;
  else
    *reinterpret_cast<u32x2 *>(static_cast<uint16_t *>(a.out) + at) =
        u32x2{round_bf16x2(v[0], v[1]), round_bf16x2(v[2], v[3])};
}

// Partials travel between workgroups by agent-scope stores and loads, eight bytes each.
__device__ __forceinline__ void leave(float *at, float x, float y) {
  __hip_atomic_store(reinterpret_cast<uint64_t *>(at),
                     (uint64_t)__float_as_uint(y) << 32 | __float_as_uint(x), __ATOMIC_RELAXED,
                     __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void pick_up(const float *at, float &x, float &y) {
  const uint64_t v = __hip_atomic_load(reinterpret_cast<const uint64_t *>(at), __ATOMIC_RELAXED,
                                       __HIP_MEMORY_SCOPE_AGENT);
  x = __uint_as_float((uint32_t)v);
  y = __uint_as_float((uint32_t)(v >> 32));
}

// Four dims of a result, from a part's sums, normalised: out, or partials if the block is
// split; lse in powers of two.
template <int KV, int D>
__device__ __forceinline__ void put4(const ChunkArgs &a, const Goal &goal, int rl, int d, f32x4 v,
                                     float lse) {
  if (goal.splits > 1) {
    const int64_t at = goal.part + rl;
    leave(a.part_o + at * D + d, v[0], v[1]);
    leave(a.part_o + at * D + d + 2, v[2], v[3]);
    if (d == 0) __hip_atomic_store(a.part_lse + at, lse, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  } else {
    int token;
    const int64_t row = row_at(a, goal.q0, goal.g, goal.base + rl, token);
    store4<KV>(a, row * D + d, v);
    if (d == 0 && a.lse) a.lse[row] = lse * kLn2;
  }
}

// The rows of a block over its parts, by the workgroup that left the last one.
template <int KV, int D>
__device__ __forceinline__ void merge_parts(const ChunkArgs &a, const Goal &goal) {
  constexpr int kBatch = 4;
  const int slot = goal.kind == kTall ? min(kRows * waves_of(KV, D), goal.rows) : min(kRows, goal.rows);
  for (int i = threadIdx.x; i < goal.height * (D / 4); i += blockDim.x) {
    const int r = i / (D / 4), d = i % (D / 4) * 4;
    float m = kNoMax, l = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    for (int t0 = 0; t0 < goal.splits; t0 += kBatch) {
      float lse[kBatch];
      float v[kBatch][4];
#pragma unroll
      for (int t = 0; t < kBatch; ++t) {
        const int64_t at = goal.first_part + (int64_t)min(t0 + t, goal.splits - 1) * slot + r;
        lse[t] = __hip_atomic_load(a.part_lse + at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        pick_up(a.part_o + at * D + d, v[t][0], v[t][1]);
        pick_up(a.part_o + at * D + d + 2, v[t][2], v[t][3]);
      }
#pragma unroll
      for (int t = 0; t < kBatch; ++t) {
        if (t0 + t >= goal.splits || lse[t] == -INFINITY) continue;   // (no key seen)
        const float mm = max_f(m, lse[t]), f = exp2_fast(m - mm), x = exp2_fast(lse[t] - mm);
        m = mm;
        l = l * f + x;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = (f == 0.f ? 0.f : o[e] * f) + (x == 0.f ? 0.f : v[t][e] * x);
      }
    }
    int token;
    const int64_t row = row_at(a, goal.q0, goal.g, goal.base + r, token);
    f32x4 res;
#pragma unroll
    for (int e = 0; e < 4; ++e) res[e] = l == 0.f ? 0.f : o[e] / l;
    store4<KV>(a, row * D + d, res);
    if (d == 0 && a.lse) a.lse[row] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
  }
}

// 16-byte words of LDS: queries (float32, 256 dims) or staged operands, and a team's
// results, a row of D + 4 floats each (the 4: rows begin in different banks).
template <int KV, int D> constexpr int team_words() { return waves_of(KV, D) * kRows * (D + 4) / 4; }
template <int KV, int D> constexpr int lds_words() {
  const int work = q_in_lds<KV, D>() ? waves_of(KV, D) * operands<KV, D>() * 64 : 4 * half_words<KV, D>();
  return work > team_words<KV, D>() ? work : team_words<KV, D>();
}

template <int KV, int D>
__global__ __launch_bounds__(64 * waves_of(KV, D))
__attribute__((amdgpu_waves_per_eu(waves_of(KV, D) / 4)))
void attn_chunk_kernel(ChunkArgs a) {
  constexpr int kWaves = waves_of(KV, D);
  __shared__ __align__(16) u32x4 s_mem[lds_words<KV, D>()];
  __shared__ float s_m[kWaves][kRows], s_l[kWaves][kRows];
  __shared__ Goal s_goal[kWaves];
  __shared__ int s_last;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int hb = lane >> 5;
  Item it;
  {
    // (all wavefronts, or with solo blocks one by one, which meet at no barrier)
    Goal goal;
    if (!item_of<kWaves>(a, (int)flat_block(), wave, lane, it, goal)) return;
    s_goal[wave] = goal;                       // (scalar registers are short until the end)
  }

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
  const int64_t row = row_at(a, it.s.q0, it.g, live ? r : min(it.r0, it.s.rows - 1), token);
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

  Tiles head;
  {
    constexpr uint32_t kTile = kPage * D * elem_bytes(KV);
    head.stride = a.Hkv * kTile;
    head.k = static_cast<const char *>(a.k_pages) + (size_t)it.g * kTile;
    head.v = static_cast<const char *>(a.v_pages) + (size_t)it.g * kTile;
  }

  State<D> st;
  auto clear = [&] {
#pragma unroll
    for (int db = 0; db < D / 32; ++db) st.o[db] = zero16();
    st.ref = kNoMax;
    st.sum = 0.f;
  };
  clear();
  if (w.j0 < w.j1) {
    // whether all pages are in the pool
    bool fine = true;
    for (int j = w.j0 + (lane >> 1); j < w.j1; j += 32) {
      const int e = 2 * w.step(j) + (lane & 1);
      fine &= e >= w.pages || in_pool(a, w.table[e]);
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
      if (it.kind == kTall && fine) {
        // whole stages; those that start beyond what the block's last 32 rows all see are
        // nobody's
        constexpr int kStage = stage_steps<D>();
        ja = w.j0 + (ja - w.j0 + kStage - 1) / kStage * kStage;
        jb = max(ja, w.j0 + (jb - w.j0) / kStage * kStage);
        const int last = token_of(a, it.last_rows);
        const int end = min(w.j1, max(0, it.s.len - it.s.n + last + 1) / kKeys - w.shift);
        walk_staged<KV, D, kWaves>(st, a, w, q, head, opaque(lane), end, ja, jb, s_mem, wave);
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
        walk_plain<KV, D>(st, a, w, q, head, opaque(lane), see, ja, jb);
      if (w.j0 < w.j1) walk_masked<KV, D>(st, a, w, q, head, opaque(lane), see, ja, jb);
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
  if (see.hi == 0) {
    st.sum = 0.f;
    st.ref = kNoMax;
  }

  Goal goal = s_goal[wave];
  goal.splits = __builtin_amdgcn_readfirstlane(goal.splits);
  goal.kind = (Kind)__builtin_amdgcn_readfirstlane(goal.kind);

  // ---- a wavefront's rows ---------------------------------------------------------
  if (goal.kind != kTeam) {
    if (live) {
      const float inv = st.sum == 0.f ? 0.f : 1.f / st.sum;
      const float lse = st.sum == 0.f ? -INFINITY : st.ref + log2f(st.sum);
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          f32x4 v;
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = st.sum == 0.f ? 0.f : st.o[db][4 * y + e] * inv;
          put4<KV, D>(a, goal, r - goal.base, 32 * db + 8 * y + 4 * hb, v, lse);
        }
    }
  } else {
    // ---- a team's: sums of its wavefronts, in LDS -----------------------------------
    constexpr int kLine = D + 4;
    float *part = reinterpret_cast<float *>(s_mem);
    const int rr = lane & 31;
    if (q_in_lds<KV, D>()) __syncthreads();    // (the queries have been read)
    if (live) {
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          f32x4 v;
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = st.o[db][4 * y + e];
          *reinterpret_cast<f32x4 *>(part + (wave * goal.height + rr) * kLine + 32 * db + 8 * y + 4 * hb) = v;
        }
      s_m[wave][rr] = st.ref;                  // (both lanes of a row: the same)
      s_l[wave][rr] = st.sum;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < goal.height * (D / 4); i += 64 * kWaves) {
      const int rl = i / (D / 4), d = i % (D / 4) * 4;
      float m = s_m[0][rl];
#pragma unroll
      for (int t = 1; t < kWaves; ++t) m = max_f(m, s_m[t][rl]);
      float l = 0.f;
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int t = 0; t < kWaves; ++t) {
        const float f = exp2_fast(s_m[t][rl] - m);
        const f32x4 x = *reinterpret_cast<const f32x4 *>(part + (t * goal.height + rl) * kLine + d);
        l += s_l[t][rl] * f;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] += f == 0.f ? 0.f : x[e] * f;
      }
      f32x4 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = l == 0.f ? 0.f : o[e] / l;
      put4<KV, D>(a, goal, rl, d, v, l == 0.f ? -INFINITY : m + log2f(l));
    }
  }
  if (goal.splits == 1) return;
  if (last_arrival_of(a.tickets + (size_t)goal.ticket * kTicketStride, goal.splits, &s_last))
    merge_parts<KV, D>(a, goal);
}

template <int KV, int D>
void launch_d(const ChunkArgs &a, hipStream_t s) {
  constexpr int kWaves = waves_of(KV, D);
  const dim3 grid((unsigned)std::min<long long>(a.grid, kAlongX), 1,
                  (unsigned)((a.grid + kAlongX - 1) / kAlongX));
  if (a.map && a.batch <= 64)
    hipLaunchKernelGGL(chunk_plan_small_kernel<kWaves>, dim3(1), dim3(64), 0, s, a);
  else if (a.map)
    hipLaunchKernelGGL(chunk_plan_kernel<kWaves>, dim3(1), dim3(kScanThreads), 0, s, a);
  hipLaunchKernelGGL((attn_chunk_kernel<KV, D>), grid, dim3(64 * kWaves), 0, s, a);
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

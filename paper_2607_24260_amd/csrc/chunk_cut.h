// How kap_chunk_attention's work is cut: what the host allows for (plan_chunk: workgroups,
// counters, rows of partial results) and the cut that the device makes of the lengths it
// finds, which has to keep to that. For the host too: nothing here needs a wavefront.
#pragma once

#include "attn_tiles.h"

#include <algorithm>

namespace kap {

constexpr int kRows = 32;                      // of a wavefront
constexpr int kKeys = 32;                      // of a step

// How the rows of a sequence are taken:
//   tall: in blocks of 32 rows a wavefront, a workgroup's wavefronts over the same steps;
//   team: in blocks of 32, a workgroup's wavefronts sharing the steps;
//   solo: in blocks of 32, a wavefront by itself.
// The steps of tall and team blocks may be split over several workgroups (parts), the last
// of which merges what they leave.
enum Kind { kTall, kTeam, kSolo };

// A sequence's part in a call.
struct Seq {
  int q0, n, len;    // first row of q, new tokens, length
  int rows;          // n * G
};
__host__ __device__ __forceinline__ Seq seq_of(const ChunkArgs &a, int b) {
  Seq s;
  s.q0 = clamp_to(a.q_offsets[b], 0, a.num_tokens);
  s.n = clamp_to(a.q_offsets[b + 1], s.q0, a.num_tokens) - s.q0;
  s.len = clamp_to(a.seq_lens[b], 0, a.max_len);
  s.rows = s.n * a.G;
  return s;
}

// r / G for 0 <= r < 2^31, given 1 / G to double precision: within one, then mended.
__host__ __device__ __forceinline__ int token_of(const ChunkArgs &a, int r) {
  int q = (int)((double)r * a.rcp_g);
  const int rest = r - q * a.G;
  q += rest >= a.G ? 1 : 0;
  q -= rest < 0 ? 1 : 0;
  return q;
}

// Steps that rows [r0, r1) of a sequence walk: the first `sinks` of them, then those
// from `from` on.
struct Range {
  int sinks, from, steps;
};
__host__ __device__ __forceinline__ Range range_of(const ChunkArgs &a, const Seq &s, int r0, int r1) {
  const int p0 = s.len - s.n + token_of(a, r0), p1 = s.len - s.n + token_of(a, r1 - 1);
  Range r;
  const int hi = max(0, p1 + 1);
  // (rows before position 0 see nothing; less a window of nearly 2^31 they would wrap)
  const int lo = a.window > 0 ? max(0, max(p0, 0) - a.window + 1) : 0;
  r.from = min(lo, hi) / kKeys;
  r.sinks = min((min(a.sinks, hi) + kKeys - 1) / kKeys, r.from);
  r.steps = r.sinks + (hi + kKeys - 1) / kKeys - r.from;
  return r;
}
__host__ __device__ __forceinline__ Range block_range(const ChunkArgs &a, const Seq &s, int size, int block) {
  return range_of(a, s, block * size, min((block + 1) * size, s.rows));
}

// What the cut goes by: a sequence's blocks, and the steps of one, on average and at most,
// in blocks of 32 rows and in tall ones.
struct Steps {
  int blocks;
  float mean, most;
};
struct Info {
  int n, rows;
  Steps by32, tall;
};
__host__ __device__ __forceinline__ Steps steps_of(const ChunkArgs &a, const Seq &s, int size) {
  Steps f{(s.rows + size - 1) / size, 0.f, 0.f};
  if (f.blocks > 0) {
    const float x = (float)block_range(a, s, size, 0).steps;
    const float y = (float)block_range(a, s, size, f.blocks - 1).steps;
    f.mean = 0.5f * (x + y);
    f.most = fmaxf(x, y);
  }
  return f;
}
template <int WAVES>
__host__ __device__ __forceinline__ Info info_of(const ChunkArgs &a, const Seq &s) {
  return Info{s.n, s.rows, steps_of(a, s, kRows), steps_of(a, s, kRows * WAVES)};
}

template <class T> __host__ __device__ __forceinline__ T pick(bool c, T x, T y) { return c ? x : y; }

// The cut: whether every sequence goes to teams, which ones to wavefronts by themselves, and
// the steps of a tall part and of a team's.
struct Cut {
  bool small;
  float solo;                  // blocks of up to so many steps go to wavefronts by themselves
  float tall_len, team_len;
  __host__ __device__ __forceinline__ Kind kind(const ChunkArgs &a, const Info &f) const {
    if (!small && f.rows > a.few_rows) return kTall;
    return f.by32.most <= solo ? kSolo : kTeam;
  }
  __host__ __device__ __forceinline__ int splits(Kind k, const Info &f) const {
    if (k == kSolo) return 1;
    const float most = pick(k == kTall, f.tall.most, f.by32.most);
    const float l = pick(k == kTall, tall_len, team_len);
    return l >= most ? 1 : (int)ceilf(most / l);
  }
};

// Steps of a sequence's longest part.
__host__ __device__ __forceinline__ float part_steps(const Cut &c, Kind k, const Info &f) {
  return pick(k == kTall, f.tall.most, f.by32.most) / (float)c.splits(k, f);
}

// Small calls go to teams throughout: a tall block's rows would leave most of the device
// idle. Blocks are split so that all parts run at once, as long as each other as near as the
// costs of steps say, or fill as many rounds as the blocks need, or to a half, a third, ..
// of the longest, if that is expected to end earlier. Parts about as long as each other end in
// rounds; others with the work over the workgroups that run at once, and half a part more,
// for which some of them idle. (Costs in eighths of a microsecond: a part 15 us around its
// steps; each part that splitting adds 15 more, or 45 in a call with tall blocks, whose parts
// leave 256 rows: a 1024-token prompt 47 us whole, 67 in halves, 700 tokens 39 and 73. Teams'
// parts of such a call, of 32 rows, are charged the 45 too: single tokens beside a prompt are
// split less than by themselves. 48 single tokens and four chunks of 512 at 8192: 311 us
// unsplit, 365 with all split to fill the rounds, 290 as expected here and longest first.)
//   sum(f), most(f): that of f(Info) of all sequences, in single precision: every wavefront
// that computes it finds the same.
constexpr float kPartCost = 120.f, kTallSplitCost = 360.f;

//   ROUNDS: there may be more blocks than workgroups that run at once.
template <int WAVES, bool ROUNDS, class Sum, class Most>
__host__ __device__ __forceinline__ Cut cut_of(const ChunkArgs &a, Sum sum, Most greatest) {
  const float Hkv = (float)a.Hkv, target = (float)a.target;
  Cut c;
  const long long tokens = sum([](const Info &f) { return f.n; });
  const float blocks = sum([](const Info &f) { return (float)f.by32.blocks; }) * Hkv;
  const float steps = sum([](const Info &f) { return (float)f.by32.blocks * f.by32.mean; }) * Hkv;
  c.small = blocks <= 2.f * target && steps <= 8.f * target * WAVES;
  // (many blocks: those no longer than about a wavefront's share of them all)
  c.solo = -1.f;
  if constexpr (ROUNDS) {
    auto few = [&](const Info &f) { return f.rows <= a.few_rows ? (float)f.by32.blocks : 0.f; };
    if (sum(few) * Hkv > 2.f * target)
      c.solo = fmaxf(8.f, 1.25f * sum([&](const Info &f) { return few(f) * f.by32.mean; }) * Hkv /
                              (target * WAVES));
  }
  const float tall_cost = (float)a.tall_cost, team_cost = (float)a.team_cost;
  const float total = sum([&](const Info &f) {
    const bool tall = c.kind(a, f) == kTall;
    return tall ? (float)f.tall.blocks * f.tall.mean * tall_cost
                : (float)f.by32.blocks * f.by32.mean * team_cost;
  }) * Hkv;
  float split_cost = kPartCost;
  if constexpr (ROUNDS) {
    if (sum([&](const Info &f) { return c.kind(a, f) == kTall ? 1.f : 0.f; }) > 0.f)
      split_cost = kTallSplitCost;
  }
  auto groups = [&](const Info &f) {
    const Kind k = c.kind(a, f);
    return (float)pick(k == kTall, f.tall.blocks, f.by32.blocks) * (float)c.splits(k, f) *
           (k == kSolo ? 1.f / WAVES : 1.f);
  };
  auto cut_to = [&](float per) {               // workgroups, with parts of that cost
    c.tall_len = fmaxf(ceilf(per / tall_cost), (float)a.tall_least);
    c.team_len = fmaxf(ceilf(per / team_cost), (float)a.team_least);
    return sum(groups) * Hkv;
  };
  const float whole = 1e9f, least = cut_to(whole);
  float best = whole;
  // (nothing is split: with more tokens than there are, as offsets say that do not ascend;
  // or where the float counts below would not be exact, and the counters' number relies on them)
  if (tokens <= a.num_tokens && total > 0.f && least <= 1048576.f) {
    // the most rounds that are full with what fits them
    const float most = ceilf(fmaxf(least / target, 1.f)) * target;
    float per = fmaxf(total / most, 1.f), n = cut_to(per);
    for (int i = 0; i < 4 && n > most; ++i) {
      per *= fmaxf(n / most, 1.05f);
      n = cut_to(per);
    }
    if constexpr (!ROUNDS) {
      if (n <= most) return c;
    } else {
      const float bound = least + 2.f * target;
      float time = 1e30f, longest = 0.f;
      // cut to parts of `per`: if it is expected to end earlier
      auto try_out = [&](float per) {
        const float n = cut_to(per), mean = total / n;
        const float part = greatest([&](const Info &f) {
          const Kind k = c.kind(a, f);
          return part_steps(c, k, f) * pick(k == kTall, tall_cost, team_cost);
        });
        if (per == whole) longest = part;
        float t;
        if (n <= target) t = part + kPartCost + (n > least ? split_cost : 0.f);
        else
          t = (kPartCost * n + split_cost * (n - least)) / target +
              (part <= 1.25f * mean ? ceilf(n / target) * part : total / target + 0.5f * mean);
        if (n <= bound && t < time) {
          time = t;
          best = per;
        }
      };
      try_out(whole);
      if (n <= most) try_out(per);
      for (int i = 2; i <= 4; ++i) try_out(longest / (float)i);
    }
  }
  cut_to(best);
  return c;
}

// Parts of a sequence, blocks that are merged, rows of partials.
struct Parts {
  int splits, parts, merges;
  long long rows;
};
template <int WAVES>
__host__ __device__ __forceinline__ Parts parts_of(const ChunkArgs &a, const Cut &c, const Info &f) {
  const Kind k = c.kind(a, f);
  Parts p;
  p.splits = c.splits(k, f);
  const int blocks = pick(k == kTall, f.tall.blocks, f.by32.blocks) * a.Hkv;
  p.parts = blocks * p.splits;
  p.merges = p.splits > 1 ? blocks : 0;
  p.rows = p.splits > 1 ? (long long)p.parts * min(k == kTall ? kRows * WAVES : kRows, f.rows) : 0;
  return p;
}
// Workgroups take tall parts and teams' alternately, in proportion, eight at a time (one of
// each XCD): the ones keep the matrix units busy, the others the memory (48 tokens and four
// chunks: 299 us, 360 one kind after the other). Solo blocks come
// last. Workgroup w's kind, and in w its place among the parts of that kind.
__host__ __device__ __forceinline__ int place(int tall, int team, int waves, int wave, int &w) {
  const int nt = (tall + 7) / 8, nm = (team + 7) / 8, group = w >> 3;
  if (group >= nt + nm) {
    w = (w - 8 * (nt + nm)) * waves + wave;
    return kSolo;
  }
  const int before = nt == 0 ? 0 : (nm == 0 ? group : (int)((long long)group * nt / (nt + nm)));
  const bool is_tall = nm == 0 || (nt > 0 && (int)((long long)(group + 1) * nt / (nt + nm)) > before);
  w = (is_tall ? before : group - before) * 8 + (w & 7);
  return is_tall ? kTall : kTeam;
}

// Sizes of a call's workspace: [arrival counters][map][partial o][partial lse], and what the
// work is cut by.
struct ChunkPlan {
  int few_rows, target, tall_cost, team_cost, tall_least, team_least, window;
  bool planned;                  // the work map is made by a launch of its own
  long long grid;
  size_t map, part_o, part_lse, total;
};

inline ChunkPlan plan_chunk(int kv_type, int D, int Hq, int num_kv_heads, int batch, int num_tokens,
                            int max_seq_len, int window, int sinks, int cus) {
  auto cdiv = [](long long a, long long b) { return (a + b - 1) / b; };
  auto round_up = [](size_t x, size_t m) { return (x + m - 1) / m * m; };
  ChunkPlan p;
  const bool f32 = kv_type == kF32;
  const int waves = chunk_waves(kv_type, D), tall = 32 * waves;
  const long long Hkv = num_kv_heads;
  const long long rows = (long long)num_tokens * (Hq / Hkv);
  p.window = window > 0 && window < max_seq_len ? window : 0;
  // More rows go to tall blocks: 64 sequences of 160 rows at 1000 tokens, bf16, 128 dims, 97 us
  // so and 223 in teams, of 96 rows 80 and 127, of 124 rows 87 and 175: of many sequences those
  // of 65 to 128 rows would be faster in tall blocks too. (256-dim float32 heads have no staged
  // walk: a prompt of 1500 tokens, 16 heads over 8, 388 us, of 128 dims 161.)
  p.few_rows = f32 && D == 256 ? 0x7fffffff : 128;
  p.target = cus;
  // in eighths of a microsecond: 32 keys with all rows of a tall block, and as their
  // bytes come from memory
  p.tall_cost = std::max(1, f32 ? D * 28 / 128 : D / 16);
  p.team_cost = std::max(1, 64 * D * elem_bytes(kv_type) * 5 / 16384);
  p.tall_least = 8;
  // (16-bit and fp8: 8 to 64 steps differ by less than the exchange costs; products of float32
  // take eight times as long: one token at 2048, 128 dims 19.6 us with 4, 29.5 with 16, 256
  // dims 32 and 76)
  p.team_least = f32 ? 4 : 16;
  // workgroups: a block each, and what splitting may add
  const long long tall_blocks =
      rows <= p.few_rows ? 0 : rows / tall + std::min<long long>(batch, rows / (p.few_rows + 1ll));
  const long long few_blocks = rows / 32 + batch;
  const long long teams = p.few_rows > 128 ? few_blocks * Hkv
                                           : std::min(few_blocks * Hkv, std::max<long long>(
                                                 4ll * batch * Hkv, 2ll * p.target));
  // Workgroups find their part by themselves if a wavefront has a lane for every sequence and
  // they all run at once; else a launch before them writes a map.
  p.planned = batch > 64 || tall_blocks * Hkv + teams > p.target;
  p.grid = tall_blocks * Hkv + teams + 2ll * p.target + 16;   // (16: places by eights)
  // What is split is at most 2 target blocks and 4 target parts, each with the rows of a
  // tall block or, of teams, at most 32; and only where a block has more steps than a
  // part's least.
  long long steps = cdiv(max_seq_len, 32);
  if (p.window)
    steps = std::min<long long>(steps, cdiv(std::min(sinks, max_seq_len), 32) + 2 +
                                           ((long long)p.window + std::min(num_tokens, tall)) / 32);
  const bool splits = steps > std::min(p.tall_least, p.team_least);
  const long long parts = splits ? 4ll * p.target : 0;
  const long long part_rows =
      std::min(parts * (tall_blocks > 0 ? tall : 32), 2 * rows * Hkv * steps);
  // (as many counters for every call: one's scratch is never another's counters)
  p.map = round_up((size_t)2 * p.target * kTicketStride * sizeof(int32_t), 256);
  p.part_o = p.map + (p.planned ? round_up(48 * (size_t)batch + 16, 256) : 0);
  p.part_lse = p.part_o + round_up((size_t)part_rows * D * sizeof(float), 256);
  p.total = p.part_lse + round_up((size_t)part_rows * sizeof(float), 256);
  return p;
}

}  // namespace kap

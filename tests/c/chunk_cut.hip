// The cut of kap_chunk_attention's work, as the library's host and device code make it, for
// tests without a GPU (host code only).
#include "chunk_cut.h"

#include <type_traits>
#include <vector>

using namespace kap;

namespace {

ChunkArgs sizes(int max_len, int window, int sinks) {
  ChunkArgs a{};
  a.max_len = max_len;
  a.window = window > 0 && window < max_len ? window : 0;
  a.sinks = a.window ? std::min(sinks, max_len) : 0;
  return a;
}

// Sums as a workgroup makes them: in single precision over 64 at a time.
template <class F> float sum_of(const std::vector<Info> &f, F g) {
  float all = 0.f;
  for (size_t i = 0; i < f.size(); i += 64) {
    float x[64];
    for (size_t j = 0; j < 64; ++j) x[j] = i + j < f.size() ? (float)g(f[i + j]) : 0.f;
    for (int n = 32; n > 0; n /= 2)
      for (int j = 0; j < n; ++j) x[j] += x[j + n];
    all += x[0];
  }
  return all;
}
struct Sum {
  const std::vector<Info> &f;
  template <class F> auto operator()(F g) const -> decltype(g(f[0]) + 0) {
    if constexpr (std::is_same<decltype(g(f[0])), int>::value) {
      long long n = 0;
      for (const Info &x : f) n += g(x);
      return (int)std::min<long long>(n, 0x7fffffff);
    } else {
      return sum_of(f, g);
    }
  }
};
struct Most {
  const std::vector<Info> &f;
  template <class F> float operator()(F g) const {
    float m = 0.f;
    for (const Info &x : f) m = std::max(m, (float)g(x));
    return m;
  }
};

template <int WAVES> void cut(ChunkArgs &a, const ChunkPlan &p, int64_t *res) {
  std::vector<Info> f;
  for (int b = 0; b < a.batch; ++b) f.push_back(info_of<WAVES>(a, seq_of(a, b)));
  const Cut c = p.planned ? cut_of<WAVES, true>(a, Sum{f}, Most{f}) : cut_of<WAVES, false>(a, Sum{f}, Most{f});
  int64_t parts[3] = {0, 0, 0}, whole = 0, merged = 0, rows = 0;
  for (const Info &x : f) {
    const Kind k = c.kind(a, x);
    const Parts y = parts_of<WAVES>(a, c, x);
    parts[k] += y.parts;
    if (y.splits > 0) whole += y.parts / y.splits;
    merged += y.merges;
    rows += y.rows;
  }
  // every part has a workgroup, or a wavefront of one
  std::vector<int64_t> met[3];
  for (int k = 0; k < 3; ++k) met[k].assign(parts[k], 0);
  int64_t last = -1;
  for (int64_t w = 0; w < p.grid; ++w)
    for (int wave = 0; wave < WAVES; ++wave) {
      int at = (int)w;
      const int k = place((int)parts[0], (int)parts[1], WAVES, wave, at);
      if ((k == kSolo || wave == 0) && at < parts[k]) {
        ++met[k][at];
        last = w;
      }
    }
  int64_t wrong = 0;
  for (int k = 0; k < 3; ++k)
    for (int64_t n : met[k]) wrong += n != 1;
  const int64_t all[] = {p.planned, parts[0], parts[1], parts[2], whole, merged, rows, wrong, last, p.grid,
                         2 * p.target, (int64_t)((p.part_lse - p.part_o) / (sizeof(float) * a.D)),
                         (int64_t)((p.total - p.part_lse) / sizeof(float))};
  static_assert(sizeof(all) / sizeof(all[0]) == 13, "");
  std::copy(all, all + 13, res);
}

}  // namespace

extern "C" {

// {sinks, from, steps} of rows [r0, r1).
void chunk_range(int n, int len, int G, int max_len, int window, int sinks, int r0, int r1, int *res) {
  ChunkArgs a = sizes(max_len, window, sinks);
  a.G = G;
  a.rcp_g = 1.0 / G;
  const Range r = range_of(a, Seq{0, n, len, n * G}, r0, r1);
  res[0] = r.sinks;
  res[1] = r.from;
  res[2] = r.steps;
}

void chunk_cut(int kv, int D, int Hq, int Hkv, int batch, int num_tokens, const int *q_offsets,
               const int *seq_lens, int max_len, int window, int sinks, int cus, int64_t *res) {
  const ChunkPlan p = plan_chunk(kv, D, Hq, Hkv, batch, num_tokens, max_len, window, sinks, cus);
  ChunkArgs a = sizes(max_len, window, sinks);
  a.batch = batch;
  a.num_tokens = num_tokens;
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.G = Hq / Hkv;
  a.D = D;
  a.rcp_g = 1.0 / a.G;
  a.q_offsets = q_offsets;
  a.seq_lens = seq_lens;
  a.few_rows = p.few_rows;
  a.target = p.target;
  a.tall_cost = p.tall_cost;
  a.team_cost = p.team_cost;
  a.tall_least = p.tall_least;
  a.team_least = p.team_least;
  if (chunk_waves(kv, D) == 4) cut<4>(a, p, res);
  else cut<8>(a, p, res);
}

}

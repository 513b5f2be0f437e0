// KV append with the position rotation applied on the way (the slot-mapped
// append of Sec. 3.1 / 3.2, KV^{full,+}, for keys and queries as the projection
// leaves them): one launch turns Q and K of the new tokens by their positions,
// writes Q out and K and V into their pages.
//
// Frequency j < rot / 2 of token t turns one pair (x, y) of dims by
//   a = positions[axis(j)][t] * inv_freq[j]:  (x cos a - y sin a, y cos a + x sin a),
// the pair being dims (j, j + rot / 2) or (2 j, 2 j + 1). The product and its
// remainder after whole quarter turns are taken in 64 bits: at position 2^18 a
// 32-bit angle is off by up to 2^-7. Sine and cosine of what is left, and the
// rotation, are 32-bit.
//
// Bound by memory: every element is read once and written once. 8192 tokens of 32
// query and 8 KV heads of 128 dims, bf16 (201 MB): 41.1 us, 4.9 TB/s, which is what a
// copy of that size reaches; the angles are not seen in it.
// float32, 3711 tokens of 16 and 8 heads of 64 dims (61 MB): 14.9 us, 4.1 TB/s. A few
// tokens are bound by the launch and by chains of a few reads: 320 tokens with fp8
// pages 7.8 us (7.0 without the angles, 0.15 less without the scales, which wait for
// the slots), one token 4.3 us.
//
// A workgroup is a role (Q heads, K heads, V columns) of a tile of 16 tokens. The
// workgroups that an XCD is given one after the other are the roles of one tile: Q's
// rows are then read and written in one sweep (51 us when a role went over all tiles
// first, 8192 tokens) and each XCD has as many of each role.
#include "kap_internal.h"

#include <algorithm>
#include <type_traits>

namespace kap {
namespace {

constexpr int kThreads = 256;
// Rows from here on (more than an L2's 4 MB) are not kept in the caches: 8192 tokens
// 48.2 -> 42.5 us, 1024 tokens 12.5 -> 10.8 us, 512 tokens 9.4 -> 9.0 us; below there
// is no difference, and what reads Q next may find it in an L2. float32 rows are kept:
// a chunk of theirs is two stores, which the caches join (16 -> 25 us without).
constexpr long long kOnceBytes = 4 << 20;
// Workgroups to reach before a thread takes more than one head (320 tokens: 9.9 us
// with four heads a thread, 8.1 us with one; 8192 tokens 62.8 us with two, 61.2 us
// with four, 59.7 us with eight, then more registers than pay elsewhere).
constexpr long long kFull = 512;
// Heads whose loads a thread has in flight.
constexpr int kHeads = 4;
// Rows: at any address; 16-byte loads; those, and without a place in the caches kept
// for what is not used again here.
constexpr int kUnaligned = 0, kAligned = 1, kOnce = 2;

template <int KV> using In = typename std::conditional<KV == kF32, uint32_t, uint16_t>::type;
template <int KV>
using Out = typename std::conditional<
    KV == kF32, uint32_t, typename std::conditional<KV == kBF16, uint16_t, uint8_t>::type>::type;

// Eight consecutive values as they lie in memory (16-byte loads where every row
// is aligned for them).
template <int KV> struct Raw8 { kv_u32x4 r[KV == kF32 ? 2 : 1]; };

template <int KV, int MODE>
__device__ __forceinline__ Raw8<KV> load8(const In<KV> *p) {
  Raw8<KV> x;
  if constexpr (MODE == kOnce) {
    x.r[0] = __builtin_nontemporal_load(reinterpret_cast<const kv_u32x4 *>(p));
  } else if constexpr (MODE == kAligned) {
    x.r[0] = reinterpret_cast<const kv_u32x4 *>(p)[0];
    if constexpr (KV == kF32) x.r[1] = reinterpret_cast<const kv_u32x4 *>(p)[1];
  } else if constexpr (KV == kF32) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x.r[i >> 2][i & 3] = p[i];
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) x.r[0][i] = p[2 * i] | (uint32_t)p[2 * i + 1] << 16;
  }
  return x;
}

template <int KV>
__device__ __forceinline__ void widen8(const Raw8<KV> &x, float v[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if constexpr (KV == kF32) v[i] = __uint_as_float(x.r[i >> 2][i & 3]);
    else v[i] = (i & 1) ? bf16_hi(x.r[0][i >> 1]) : bf16_lo(x.r[0][i >> 1]);
  }
}

// In the type they came in, rounded once (nearest even).
template <int KV, int MODE>
__device__ __forceinline__ void store8(void *p, const float v[8]) {
  kv_u32x4 *d = static_cast<kv_u32x4 *>(p);
  if constexpr (KV == kF32) {
    d[0] = kv_u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]),
                    __float_as_uint(v[3])};
    d[1] = kv_u32x4{__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]),
                    __float_as_uint(v[7])};
  } else {
    const kv_u32x4 x = {round_bf16x2(v[0], v[1]), round_bf16x2(v[2], v[3]),
                        round_bf16x2(v[4], v[5]), round_bf16x2(v[6], v[7])};
    if constexpr (MODE == kOnce) __builtin_nontemporal_store(x, d);
    else *d = x;
  }
}

// x / scale as an E4M3FN code: nearest even, +-448 beyond the range, NaN kept.
__device__ __forceinline__ float fp8_range(float x, float scale) {
  const float y = x / scale;
  return y > 448.f ? 448.f : (y < -448.f ? -448.f : y);
}
__device__ __forceinline__ uint32_t fp8_codes(float x0, float x1, float x2, float x3, float s) {
  const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(fp8_range(x0, s), fp8_range(x1, s), 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(fp8_range(x2, s), fp8_range(x3, s), lo, true);
}

// Chunk c (eight dims) of KV head g of the token in `off` of a page.
template <int KV, int MODE>
__device__ __forceinline__ void store_k(const RopeAppendArgs &a, int64_t page, int off, int g,
                                        int c, float scale, const float v[8]) {
  Out<KV> *d = static_cast<Out<KV> *>(a.k_pages) +
               (((size_t)page * a.Hkv + g) * (a.D / 8) + c) * (kPage * 8) + off * 8;
  if constexpr (KV == kFP8) {
    *reinterpret_cast<kv_u32x2 *>(d) = kv_u32x2{fp8_codes(v[0], v[1], v[2], v[3], scale),
                                                fp8_codes(v[4], v[5], v[6], v[7], scale)};
  } else {
    store8<KV, MODE>(d, v);
  }
}

// (cos a, sin a), a = pos * freq: whole quarter turns are taken off in 64 bits.
__device__ __forceinline__ float2 turn_of(int pos, float freq) {
  const double quarters = (double)pos * (double)freq * 0.63661977236758134308;   // 2 / pi
  const double whole = rint(quarters);
  float s, c;
  sincospif((float)(quarters - whole) * 0.5f, &s, &c);
  const int n = (int)(long long)(whole - 4.0 * floor(whole * 0.25));
  if (n & 1) {
    const float t = s;
    s = c;
    c = -t;
  }
  if (n & 2) {
    s = -s;
    c = -c;
  }
  return make_float2(c, s);
}

// (x, y) turned. An angle of 0 leaves both as they are, next to an infinity or NaN too
// (which the product with a sine of 0 would make NaN).
__device__ __forceinline__ void turn(float x, float y, float2 cs, float &p, float &q) {
  const float xc = x * cs.x, yc = y * cs.x;
  p = cs.y == 0.f ? xc : fmaf(-y, cs.y, xc);
  q = cs.y == 0.f ? yc : fmaf(x, cs.y, yc);
}

// Rows of Q (chunks in neighbouring lanes: 128 and more contiguous bytes of a
// row per token), or of K (tokens in neighbouring lanes: a page holds a chunk's
// 16 tokens side by side). A thread has one chunk pair of one token -- eight
// frequencies, in registers -- and goes over heads with it.
template <int KV, int MODE>
__device__ __forceinline__ void rotate_rows(const RopeAppendArgs &a, int bx, bool is_k, int slice,
                                            float2 *s_cs) {
  const int t0 = bx * a.tile, nt = min(a.tile, a.num_tokens - t0);
  const int nf = a.rot / 2, P = a.rot / 16;
  const int per_head = P * a.tile, hs_n = kThreads / per_head;
  const int hs = threadIdx.x / per_head, rem = threadIdx.x - hs * per_head;
  const int tok = is_k ? rem % a.tile : rem / P;
  const int c = is_k ? rem / a.tile : rem - tok * P;
  const int H = is_k ? a.Hkv : a.Hq;
  const int h0 = slice * hs_n * a.heads, h1 = min(H, h0 + hs_n * a.heads);
  const In<KV> *src = static_cast<const In<KV> *>(is_k ? a.k_new : a.q_new);
  const size_t stride = (size_t)(is_k ? a.k_stride : a.q_stride);
  const bool mine = hs < hs_n && tok < nt;
  const int ca = a.halves ? c : 2 * c, cb = a.halves ? c + P : 2 * c + 1;

  Raw8<KV> xa[kHeads], xb[kHeads];
  const In<KV> *row = src + (size_t)(t0 + (mine ? tok : 0)) * stride;
#pragma unroll
  for (int u = 0; u < kHeads; ++u) {
    const int h = h0 + hs + u * hs_n;
    if (mine && h < h1) {
      xa[u] = load8<KV, MODE>(row + (size_t)h * a.D + ca * 8);
      xb[u] = load8<KV, MODE>(row + (size_t)h * a.D + cb * 8);
    }
  }
  const int64_t most = a.num_pages * kPage;
  auto slot_of = [&](int t) {                  // -1: nothing to write
    const int64_t s = a.slots[t0 + t];
    return s < most ? s : -1;
  };
  const int64_t slot = is_k && mine ? slot_of(tok) : 0;
  const float scale = KV == kFP8 && is_k && mine && slot >= 0 ? a.kv_scales[2 * (slot / kPage)] : 1.f;

  for (int i = threadIdx.x; i < nt * nf; i += kThreads) {
    const int t = i / nf, j = i - t * nf;
    const int axis = a.freq_axis ? a.freq_axis[j] : 0;
    // an axis that is not there turns nothing (position and frequency are loaded for it
    // too: 8192 tokens 41.1 us, 41.9 with branches around the loads)
    const bool there = axis >= 0 && axis < a.num_axes;
    const int pos = a.positions[(size_t)(there ? axis : 0) * a.num_tokens + t0 + t];
    const float freq = a.inv_freq[j];
    s_cs[i] = there ? turn_of(pos, freq) : make_float2(1.f, 0.f);
  }
  __syncthreads();
  if (mine && slot >= 0) {
    float2 cs[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) cs[i] = s_cs[tok * nf + 8 * c + i];
#pragma unroll
    for (int u = 0; u < kHeads; ++u) {
      const int h = h0 + hs + u * hs_n;
      if (h >= h1) continue;
      float x[8], y[8], p[8], q[8];
      widen8<KV>(xa[u], x);
      widen8<KV>(xb[u], y);
      if (a.halves) {
#pragma unroll
        for (int i = 0; i < 8; ++i) turn(x[i], y[i], cs[i], p[i], q[i]);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          turn(x[2 * i], x[2 * i + 1], cs[i], p[2 * i], p[2 * i + 1]);
          turn(y[2 * i], y[2 * i + 1], cs[4 + i], q[2 * i], q[2 * i + 1]);
        }
      }
      if (is_k) {
        const int64_t page = slot / kPage;
        const int off = (int)(slot - page * kPage);
        store_k<KV, MODE>(a, page, off, h, ca, scale, p);
        store_k<KV, MODE>(a, page, off, h, cb, scale, q);
      } else {
        In<KV> *dst = static_cast<In<KV> *>(a.q_out) + ((size_t)(t0 + tok) * a.Hq + h) * a.D;
        store8<KV, MODE>(dst + ca * 8, p);
        store8<KV, MODE>(dst + cb * 8, q);
      }
    }
  }
  // the dims that are not rotated
  const int R = (a.D - a.rot) / 8;
  const int heads = h1 - h0;
  for (int i = threadIdx.x; i < nt * R * heads; i += kThreads) {
    int t, r, h;
    if (is_k) {
      t = i % nt;
      r = i / nt % R;
      h = h0 + i / nt / R;
    } else {
      r = i % R;
      h = h0 + i / R % heads;
      t = i / R / heads;
    }
    const int ch = a.rot / 8 + r;
    float x[8];
    widen8<KV>(load8<KV, MODE>(src + (size_t)(t0 + t) * stride + (size_t)h * a.D + ch * 8), x);
    if (is_k) {
      const int64_t s = slot_of(t);
      if (s < 0) continue;
      const int64_t page = s / kPage;
      const float sc = KV == kFP8 ? a.kv_scales[2 * page] : 1.f;
      store_k<KV, MODE>(a, page, (int)(s - page * kPage), h, ch, sc, x);
    } else {
      store8<KV, MODE>(static_cast<In<KV> *>(a.q_out) + ((size_t)(t0 + t) * a.Hq + h) * a.D + ch * 8, x);
    }
  }
}

// V, which a page holds transposed. A whole page -- 16 consecutive tokens in its
// 16 slots -- belongs to the 16 tokens it starts in, wherever in them it starts:
// a lane reads its 4-byte column of all 16 tokens, turns it around in registers,
// and a store instruction covers 1 KB (through LDS). Outside whole pages (a step's
// first and last, and any with a padded token in it) four tokens in an aligned four
// of a page's slots are one store a dim, and what is left is stored element by element
// (8192 tokens, one in 64 padded: 10 us less than with all of such pages' tokens by
// element), shared out over a.v_share workgroups.
template <int KV, int MODE>
__device__ __forceinline__ void append_v(const RopeAppendArgs &a, int bx, int part, int share,
                                         kv_u32x4 (*s_rows)[256]) {
  constexpr int kColDims = KV == kF32 ? 1 : 2;
  constexpr int kUnits = KV == kFP8 ? 2 : 4;   // 16-byte units of a column's page rows
  const int lane = threadIdx.x & 63;
  const int t0 = bx * kPage;
  const int row = a.Hkv * a.D, cols = row / kColDims;
  const In<KV> *src = static_cast<const In<KV> *>(a.v_new);
  const size_t stride = (size_t)a.v_stride;

  // Lane l looks at token t0 - 16 + l: is it in the slot after the token before
  // it, on the same page; and does its page's first token start 15 such?
  const int t = t0 - kPage + lane;
  const int64_t slot = t >= 0 && t < a.num_tokens ? a.slots[t] : -1;
  const bool good = slot >= 0 && slot < a.num_pages * kPage;
  const int64_t before = __shfl_up(slot, 1, 64);
  const int off = (int)(slot & (kPage - 1));
  const unsigned long long joined =
      __ballot(lane > 0 && good && before >= 0 && slot == before + 1 && off != 0);
  const int first = lane - off;                // lane of the page's first token
  const bool whole = good && first >= 0 && first + 15 < 64 &&
                     ((joined >> first >> 1) & 0x7FFFu) == 0x7FFFu;
  const bool mine = lane >= kPage && lane < 2 * kPage;
  const unsigned long long starts = __ballot(mine && whole && off == 0);   // at most one
  // likewise four tokens in an aligned four of a page's slots
  const int four = lane - (off & 3);
  const bool in_four = good && !whole && four >= 0 && ((joined >> four >> 1) & 7u) == 7u;
  const bool shared_out = mine && good && !whole && lane % a.v_share == share;
  unsigned fours = (unsigned)(__ballot(shared_out && in_four && (off & 3) == 0) >> kPage);
  unsigned single = (unsigned)(__ballot(shared_out && !in_four) >> kPage);
  if (part == 0 && share == 0 && threadIdx.x < 64 && mine && slot >= 0 && !good && a.bad_slots)
    atomicAdd(a.bad_slots, 1);
  auto slot_at = [&](int l) {                  // slot of lane l (the same l in every lane)
    return ((int64_t)__builtin_amdgcn_readlane((int)(slot >> 32), l) << 32) |
           (uint32_t)__builtin_amdgcn_readlane((int)slot, l);
  };

  if (starts && share == 0) {
    const int f = __builtin_ctzll(starts);     // lane
    const int64_t page = slot_at(f) / kPage;
    const int token = t0 - kPage + f;
    const int col = part * kThreads + threadIdx.x;
    const float scale = KV == kFP8 ? a.kv_scales[2 * page + 1] : 1.f;
    uint32_t x[kPage] = {};
    if (col < cols) {
#pragma unroll
      for (int i = 0; i < kPage; ++i) {
        const In<KV> *p = src + (size_t)(token + i) * stride + (size_t)col * kColDims;
        if constexpr (MODE != kUnaligned || KV == kF32) x[i] = *reinterpret_cast<const uint32_t *>(p);
        else x[i] = p[0] | (uint32_t)p[1] << 16;
      }
    }
    uint32_t o[4 * kUnits];
    if constexpr (KV == kF32) {
#pragma unroll
      for (int i = 0; i < kPage; ++i) o[i] = x[i];
    } else if constexpr (KV == kBF16) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {            // tokens 2 i, 2 i + 1
        o[i] = __builtin_amdgcn_perm(x[2 * i + 1], x[2 * i], 0x05040100u);
        o[8 + i] = __builtin_amdgcn_perm(x[2 * i + 1], x[2 * i], 0x07060302u);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {            // tokens 4 i .. 4 i + 3
        o[i] = fp8_codes(bf16_lo(x[4 * i]), bf16_lo(x[4 * i + 1]), bf16_lo(x[4 * i + 2]),
                         bf16_lo(x[4 * i + 3]), scale);
        o[4 + i] = fp8_codes(bf16_hi(x[4 * i]), bf16_hi(x[4 * i + 1]), bf16_hi(x[4 * i + 2]),
                             bf16_hi(x[4 * i + 3]), scale);
      }
    }
    // (units rotated by column so that the lanes of a write spread over the banks)
    kv_u32x4 *buf = s_rows[threadIdx.x >> 6];
#pragma unroll
    for (int i = 0; i < kUnits; ++i)
      buf[kUnits * lane + ((i + (lane >> 1)) & (kUnits - 1))] =
          kv_u32x4{o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]};
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    const int col0 = part * kThreads + (threadIdx.x & ~63);   // the wavefront's first column
    kv_u32x4 *dst = reinterpret_cast<kv_u32x4 *>(static_cast<Out<KV> *>(a.v_pages) +
                                                 (size_t)page * row * kPage +
                                                 (size_t)col0 * kColDims * kPage);
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
      const int u = 64 * i + lane, c = u / kUnits;
      if (col0 + c < cols) dst[u] = buf[kUnits * c + (((u & (kUnits - 1)) + (c >> 1)) & (kUnits - 1))];
    }
  }
  // four tokens of a column in a store
  const int my_col = part * kThreads + threadIdx.x;
  while (fours) {
    constexpr int kBatch = 2;
    int token[kBatch];
    uint32_t x[kBatch][4] = {};
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      token[i] = fours ? __builtin_ctz(fours) : -1;
      fours &= fours - 1;
      if (token[i] < 0 || my_col >= cols) continue;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const In<KV> *p = src + (size_t)(t0 + token[i] + e) * stride + (size_t)my_col * kColDims;
        if constexpr (MODE != kUnaligned || KV == kF32) x[i][e] = *reinterpret_cast<const uint32_t *>(p);
        else x[i][e] = p[0] | (uint32_t)p[1] << 16;
      }
    }
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      if (token[i] < 0 || my_col >= cols) continue;
      const int64_t to = slot_at(kPage + token[i]);
      const int64_t page = to / kPage;
      Out<KV> *d = static_cast<Out<KV> *>(a.v_pages) + (size_t)page * row * kPage +
                   (size_t)my_col * kColDims * kPage + (to & (kPage - 1));
      if constexpr (KV == kF32) {
        *reinterpret_cast<kv_u32x4 *>(d) = kv_u32x4{x[i][0], x[i][1], x[i][2], x[i][3]};
      } else if constexpr (KV == kBF16) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const uint32_t sel = e ? 0x07060302u : 0x05040100u;
          *reinterpret_cast<kv_u32x2 *>(d + e * kPage) =
              kv_u32x2{__builtin_amdgcn_perm(x[i][1], x[i][0], sel),
                       __builtin_amdgcn_perm(x[i][3], x[i][2], sel)};
        }
      } else {
        const float scale = a.kv_scales[2 * page + 1];
        *reinterpret_cast<uint32_t *>(d) = fp8_codes(bf16_lo(x[i][0]), bf16_lo(x[i][1]),
                                                     bf16_lo(x[i][2]), bf16_lo(x[i][3]), scale);
        *reinterpret_cast<uint32_t *>(d + kPage) = fp8_codes(
            bf16_hi(x[i][0]), bf16_hi(x[i][1]), bf16_hi(x[i][2]), bf16_hi(x[i][3]), scale);
      }
    }
  }
  // element by element: a store instruction covers 64 neighbouring rows
  const int e0 = part * kThreads * kColDims + threadIdx.x;
  while (single) {
    constexpr int kBatch = 4;
    int token[kBatch];
    In<KV> x[kBatch][kColDims];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      token[i] = single ? __builtin_ctz(single) : -1;
      single &= single - 1;
#pragma unroll
      for (int e = 0; e < kColDims; ++e)
        if (token[i] >= 0 && e0 + e * kThreads < row)
          x[i][e] = src[(size_t)(t0 + token[i]) * stride + e0 + e * kThreads];
    }
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      if (token[i] < 0) continue;
      const int64_t to = slot_at(kPage + token[i]);
      const int64_t page = to / kPage;
      Out<KV> *dst = static_cast<Out<KV> *>(a.v_pages) + (size_t)page * row * kPage +
                     (to & (kPage - 1));
      const float scale = KV == kFP8 ? a.kv_scales[2 * page + 1] : 1.f;
#pragma unroll
      for (int e = 0; e < kColDims; ++e) {
        if (e0 + e * kThreads >= row) continue;
        Out<KV> *d = dst + (size_t)(e0 + e * kThreads) * kPage;
        if constexpr (KV == kFP8) {
          const float v = __uint_as_float((uint32_t)x[i][e] << 16);
          *d = (uint8_t)fp8_codes(v, v, v, v, scale);
        } else {
          *d = x[i][e];
        }
      }
    }
  }
}

template <int KV, int MODE>
__global__ __launch_bounds__(kThreads) void rope_append_kernel(RopeAppendArgs a) {
  __shared__ union {
    float2 cs[kPage * 128];                    // [token][frequency]
    kv_u32x4 rows[kThreads / 64][256];
  } s;
  const int xcd = blockIdx.x & 7;
  const int bx = (int)((blockIdx.x >> 3) / a.roles) * 8 + xcd;   // tile
  const int y = (int)(blockIdx.x >> 3) % a.roles;
  if (bx >= a.tiles) return;
  if (y < a.q_slices + a.k_slices) {
    const bool is_k = y >= a.q_slices;
    rotate_rows<KV, MODE>(a, bx, is_k, is_k ? y - a.q_slices : y, s.cs);
  } else {
    const int v = y - a.q_slices - a.k_slices;
    append_v<KV, MODE>(a, bx, v / a.v_share, v % a.v_share, s.rows);
  }
}

template <int KV>
void launch_kv(const RopeAppendArgs &a, unsigned grid, int mode, hipStream_t s) {
  if (mode == kUnaligned)
    hipLaunchKernelGGL((rope_append_kernel<KV, kUnaligned>), grid, dim3(kThreads), 0, s, a);
  else if (mode == kAligned || KV == kF32)
    hipLaunchKernelGGL((rope_append_kernel<KV, kAligned>), grid, dim3(kThreads), 0, s, a);
  else if constexpr (KV != kF32)
    hipLaunchKernelGGL((rope_append_kernel<KV, kOnce>), grid, dim3(kThreads), 0, s, a);
}

}  // namespace

hipError_t launch_rope_append(const RopeAppendArgs &args, hipStream_t s) {
  RopeAppendArgs a = args;
  const int es = a.kv_type == kF32 ? 4 : 2;
  const auto addr = reinterpret_cast<uintptr_t>(a.q_new) | reinterpret_cast<uintptr_t>(a.k_new) |
                    reinterpret_cast<uintptr_t>(a.v_new) |
                    (uintptr_t)((a.q_new ? a.q_stride : 0) | a.k_stride | a.v_stride) * es;
  const long long row_bytes = (long long)((a.q_new ? a.Hq : 0) + 2 * a.Hkv) * a.D * es;
  const int mode = addr % 16 != 0 ? kUnaligned
                                  : (a.num_tokens * row_bytes >= kOnceBytes ? kOnce : kAligned);
  // Tiles of 16 tokens, or of all of them, so that a few tokens' heads spread
  // over a workgroup.
  a.tile = std::min(a.num_tokens, kPage);
  a.tiles = (a.num_tokens - 1) / kPage + 1;
  const int lanes = kThreads / (a.rot / 16 * a.tile);      // heads side by side
  a.heads = kHeads;
  while (a.heads > 1 && (long long)a.tiles * ((a.Hq + a.Hkv) / (lanes * a.heads)) < kFull) a.heads /= 2;
  const int heads = a.heads * lanes;                       // of a workgroup
  a.q_slices = a.q_new ? (a.Hq + heads - 1) / heads : 0;
  a.k_slices = (a.Hkv + heads - 1) / heads;
  const int cols = a.Hkv * a.D / (a.kv_type == kF32 ? 1 : 2);
  const int parts = (cols + kThreads - 1) / kThreads;
  // Tokens outside whole pages: one workgroup that moves 16 of them one after
  // the other takes as long, so they are shared out while there are few.
  a.v_share = 1;
  while (a.v_share < kPage && 2ll * a.tiles * parts * a.v_share <= 1024) a.v_share *= 2;
  a.roles = a.q_slices + a.k_slices + parts * a.v_share;
  const long long grid = ((long long)a.tiles + 7) / 8 * 8 * a.roles;
  if (grid > 0x7fffffffll) return hipErrorInvalidValue;
  switch (a.kv_type) {
    case kF32: launch_kv<kF32>(a, (unsigned)grid, mode, s); break;
    case kBF16: launch_kv<kBF16>(a, (unsigned)grid, mode, s); break;
    default: launch_kv<kFP8>(a, (unsigned)grid, mode, s); break;
  }
  return hipGetLastError();
}

}  // namespace kap

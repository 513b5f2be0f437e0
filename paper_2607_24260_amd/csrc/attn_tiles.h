// Operands of the 32-row attention tiles on the matrix cores, as the shared-prefix
// and the chunk kernels use them: S^T[key][row] = K . Q^T and O^T[dim][row] += V^T P^T
// with 32 keys (two pages) a step.
#pragma once

#include "kap_internal.h"

namespace kap {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

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

template <class T>
__device__ __forceinline__ T wave_sum(T x) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) x += __shfl_xor(x, o, 64);
  return x;
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

__host__ __device__ __forceinline__ int clamp_to(int x, int lo, int hi) { return min(max(x, lo), hi); }

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

__device__ __forceinline__ u32x4 widen8(u32x2 x) {
  const u32x2 lo = fp8x4_to_bf16x4(x[0]), hi = fp8x4_to_bf16x4(x[1]);
  return u32x4{lo[0], lo[1], hi[0], hi[1]};
}
__device__ __forceinline__ u32x4 wide(const Operand<kBF16> &r) { return r.x; }
__device__ __forceinline__ u32x4 wide(const Operand<kF32> &r) { return r.x; }
__device__ __forceinline__ u32x4 wide(const Operand<kFP8> &r) { return widen8(r.x); }

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

}  // namespace kap

// Block tables, slots and positions of a step from its requests' lengths: pages
// that are no longer held go back to the ring of free pages, pages that the new
// tokens need come from it, and every new token gets its slot and position.
//
// Everything is prefix sums over the sequences: of the tokens asked for (which
// sequences get theirs), of the pages needed (which pages they get), of what is
// granted and returned. One workgroup takes 1024 sequences at a time, with the sums
// so far carried along (256 where that is enough: fewer wavefronts to wait for); a
// sequence's few pages are moved by its thread, many by the wavefront. There is hardly
// anything to move (12 bytes a token): what bounds a call is its chain of loads and scans,
// 4.2 us for one sequence, 5 for 64 and their 320 tokens.
//
// Slots and positions of a small step are written by the same workgroup; of a
// larger one by a second launch over all CUs. (1000 sequences of which 60 end, and eight
// prompts' 32768 tokens: 17 us, and 4.5 for the second. The pages' sequences searched for
// in the prefix sums, page by page, took 32 in all.)
#include "block_scan.h"

#include <algorithm>

namespace kap {
namespace {

constexpr int kSmall = 256;                    // sequences that a small workgroup takes
constexpr int kOwn = 4;                        // pages that a thread moves for its sequence
constexpr int kRuns = 8;                       // runs of 64 that a wavefront moves at once
constexpr int kTailThreads = 256;
constexpr int kTailOffsets = 8192;             // offsets that the second launch keeps in LDS

// Slot and position of token t of the step, the i-th new one of sequence b.
__device__ __forceinline__ void write_token(const StepArgs &a, long long t, int b, int i, int add,
                                            int new_len) {
  const int pos = new_len - add + i;
  const long long page = a.table[(size_t)b * a.stride + pos / kPage];
  a.slots[t] = page * kPage + pos % kPage;
  a.positions[t] = pos;
}
__device__ __forceinline__ void write_padding(const StepArgs &a, long long t) {
  a.slots[t] = -1;
  a.positions[t] = 0;
}

__device__ __forceinline__ long long wrapped(long long x, long long size) {
  if (x >= size) x -= size;
  return x >= size ? x - size : x;
}

// Moves n pages of each lane between its table entries and the ring's, from entry r0 on: up
// to kOwn by the lane itself, more by the wavefront, in runs of 64, several at once, of one
// lane or of several.
template <bool TAKE>
__device__ __forceinline__ void move_pages(const StepArgs &a, int n, int32_t *table, int r0) {
  const int lane = threadIdx.x & 63;
  auto ring_at = [&](int first, int i) {
    const unsigned at = (unsigned)first + (unsigned)i, size = a.ring_size;
    return a.ring + (at >= size ? at - size : at);
  };
  {
    int32_t page[kOwn];
    const bool own = n <= kOwn;
#pragma unroll
    for (int i = 0; i < kOwn; ++i)
      if (own && i < n) page[i] = TAKE ? *ring_at(r0, i) : table[i];
#pragma unroll
    for (int i = 0; i < kOwn; ++i)
      if (own && i < n) *(TAKE ? table + i : ring_at(r0, i)) = page[i];
  }
  unsigned long long left = __ballot(n > kOwn);
  const uint64_t mine = reinterpret_cast<uint64_t>(table);
  int at = 0;
  while (left) {
    int32_t page[kRuns], *to[kRuns];
    bool in[kRuns];
#pragma unroll
    for (int u = 0; u < kRuns; ++u) {
      const int l = left ? __builtin_amdgcn_readfirstlane(__ffsll((long long)left) - 1) : 0;
      const int count = left ? __builtin_amdgcn_readlane(n, l) : 0, i = at + lane;
      int32_t *const entry = reinterpret_cast<int32_t *>(
                                 (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(mine >> 32), l) << 32 |
                                 (uint32_t)__builtin_amdgcn_readlane((int)mine, l)) + i;
      in[u] = i < count;
      int32_t *const slot = ring_at(__builtin_amdgcn_readlane(r0, l), in[u] ? i : 0);
      to[u] = TAKE ? entry : slot;
      if (in[u]) page[u] = *(TAKE ? slot : entry);
      at += 64;
      if (at >= count) {
        left &= left - 1;
        at = 0;
      }
    }
#pragma unroll
    for (int u = 0; u < kRuns; ++u)
      if (in[u]) *to[u] = page[u];
  }
}

template <int kThreads>
__global__ __launch_bounds__(kThreads) void step_tables_kernel(StepArgs a) {
  constexpr int kWaves = kThreads / 64;
  __shared__ long long s_scan[3][kWaves];
  __shared__ int s_first[kThreads + 1], s_len[kThreads];
  const int tid = threadIdx.x;
  const long long size = a.ring_size;
  long long head = a.free_state[0], count = a.free_state[1];
  if (head < 0 || head >= size) head = 0;
  count = count < 0 ? 0 : (count > size ? size : count);
  long long asked = 0, wanted = 0, tokens = 0, taken = 0, returned = 0;
  for (int b0 = 0; b0 < a.batch; b0 += kThreads) {
    const int b = b0 + tid;
    const bool in = b < a.batch;
    const int len = in ? a.seq_lens[b] : 0;
    int keep = in && a.keep ? a.keep[b] : len;
    int add = in ? a.add[b] : 0;
    const int pinned = in && a.pinned ? max(a.pinned[b], 0) : 0;
    const long long room = (long long)a.stride * kPage;
    int status = kStepOk;
    const bool bad = len < 0 || keep < 0 || keep > len || add < 0 || len > room;
    if (bad) {
      status = kStepBadLength;
      keep = len;
      add = 0;
    } else if (add > 0 && (long long)keep + add > room) {
      status = kStepOverCapacity;
      add = 0;
    }
    const int have = bad ? 0 : (len + kPage - 1) / kPage;
    {
      const int x[1] = {add};
      long long incl[1], total[1];
      scan(x, incl, total, s_scan);
      if (add > 0 && asked + incl[0] > a.num_tokens) {
        status = kStepOverTokens;
        add = 0;
      }
      asked += total[0];
    }
    int need = bad ? 0 : max(0, (keep + add + kPage - 1) / kPage - have);
    {
      const int x[1] = {need};
      long long incl[1], total[1];
      scan(x, incl, total, s_scan);
      if (need > 0 && wanted + incl[0] > count) {
        status = kStepOutOfPages;
        add = need = 0;
      }
      wanted += total[0];
    }
    const int held = bad ? 0 : max((keep + add + kPage - 1) / kPage, pinned);
    const int x[3] = {add, need, max(0, have - held)};
    long long incl[3], total[3];
    scan(x, incl, total, s_scan);
    s_first[tid] = (int)(tokens + incl[0] - x[0]);
    s_len[tid] = keep + add;
    if (in) {
      a.new_lens[b] = keep + add;
      a.status[b] = status;
      a.q_offsets[b + 1] = (int)(tokens + incl[0]);
    }
    __syncthreads();
    // pages from the front of the ring, and back to its end: the first are among the
    // `count` that were there, the second go beyond them, so no entry is both
    int32_t *const row = a.table + (size_t)b * a.stride;
    move_pages<true>(a, need, row + have, (int)wrapped(head + taken + incl[1] - need, size));
    const long long before = returned + incl[2] - x[2];
    move_pages<false>(a, (int)min((long long)x[2], max(size - count - before, 0ll)), row + held,
                      (int)wrapped(head + count + min(before, size), size));
    tokens += total[0];
    taken += total[1];
    returned += total[2];
  }
  if (tid == 0) {
    a.q_offsets[0] = 0;
    a.free_out[0] = (int)wrapped(head + taken, size);
    a.free_out[1] = (int)(count - taken + (returned < size - count ? returned : size - count));
    s_first[kThreads] = (int)tokens;
  }
  if (!a.tokens_here) return;
  __syncthreads();                             // (table entries, by threads of this workgroup)
  for (int t = tid; t < a.num_tokens; t += kThreads) {
    if (t >= tokens) {
      write_padding(a, t);
      continue;
    }
    const int j = last_at_most(s_first, a.batch, t);
    const int end = j + 1 < a.batch ? s_first[j + 1] : (int)tokens;
    write_token(a, t, j, t - s_first[j], end - s_first[j], s_len[j]);
  }
}

__global__ __launch_bounds__(kTailThreads) void step_slots_kernel(StepArgs a) {
  __shared__ int s_first[kTailOffsets];
  const int *first = a.q_offsets;
  if (a.batch < kTailOffsets) {
    for (int i = threadIdx.x; i <= a.batch; i += kTailThreads) s_first[i] = a.q_offsets[i];
    __syncthreads();
    first = s_first;
  }
  const int tokens = first[a.batch];
  for (long long t = (long long)blockIdx.x * kTailThreads + threadIdx.x; t < a.num_tokens;
       t += (long long)gridDim.x * kTailThreads) {
    if (t >= tokens) {
      write_padding(a, t);
      continue;
    }
    const int b = last_at_most(first, a.batch, t);
    write_token(a, t, b, (int)t - first[b], first[b + 1] - first[b], a.new_lens[b]);
  }
}

}  // namespace

hipError_t launch_step_tables(StepArgs a, int cus, hipStream_t s) {
  // Slots of a step of up to 4096 tokens are written by the first launch, if its threads hold
  // all sequences' offsets.
  const bool small = a.batch <= kSmall;
  a.tokens_here = a.batch <= kScanThreads && a.num_tokens <= 4 * (small ? kSmall : kScanThreads);
  if (small)
    hipLaunchKernelGGL(step_tables_kernel<kSmall>, dim3(1), dim3(kSmall), 0, s, a);
  else
    hipLaunchKernelGGL(step_tables_kernel<kScanThreads>, dim3(1), dim3(kScanThreads), 0, s, a);
  if (!a.tokens_here && a.num_tokens > 0) {
    const int blocks = (a.num_tokens + kTailThreads - 1) / kTailThreads;
    hipLaunchKernelGGL(step_slots_kernel, dim3(std::min(blocks, 4 * cus)), dim3(kTailThreads), 0, s, a);
  }
  return hipGetLastError();
}

}  // namespace kap

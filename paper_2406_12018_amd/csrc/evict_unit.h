// Eviction by accumulated attention weight, of one unit by one workgroup: for the kernels that stream the unit's keys, and for one behind
// them.
//
//   w_j = sum over the heads of the group of exp2(s_j - lse),   sum_j += w_j
// and the state with the smallest sum makes room for the token's.
#pragma once

#include "few_rows.h"

namespace citrus {
namespace {

// The state that goes: the smaller sum, of equal ones the lower slot.  A sum that is not a number is never the smaller one.
struct Candidate {
  float sum;
  int slot;
};
__device__ inline Candidate smaller(const Candidate& a, const Candidate& b) {
  return b.sum < a.sum || (b.sum == a.sum && b.slot < a.slot) ? b : a;
}
__device__ inline bool may_go(const EvictStep& e, int slot) {
  return (slot >= e.start && slot < e.n - e.recent) || slot == e.oldest;
}
// scratch: a Candidate per wave; the workgroup is in step on return
template <int THREADS>
__device__ inline Candidate smallest_of_block(Candidate c, Candidate* scratch) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) c = smaller(c, Candidate{__shfl_xor(c.sum, o, 64), __shfl_xor(c.slot, o, 64)});
  if (threadIdx.x % 64 == 0) scratch[threadIdx.x / 64] = c;
  __syncthreads();
  c = scratch[0];
#pragma unroll
  for (int w = 1; w < THREADS / 64; ++w) c = smaller(c, scratch[w]);
  return c;
}

// Sums of the keys [begin, end) of a unit grow, four keys a thread and turn; begin is a multiple of 4.  scores: [head][score_pitch],
// lse2: by head.  Returns this thread's smallest; own: the token's weight, to the thread whose key it is.
template <int THREADS>
__device__ inline Candidate grow_sums(const EvictStep& e, const float* scores, int64_t pitch, const float* lse2, float* acc, int begin, int end,
                                      float* own) {
  const int G = e.dm.G;
  Candidate best{INFINITY, e.oldest};
  for (int j = begin + 4 * threadIdx.x; j < end; j += 4 * THREADS) {
    float old[4], w[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int x = 0; x < 4; ++x) old[x] = acc[min(j + x, e.n - 1 > 0 ? e.n - 1 : 0)];
#pragma unroll 4
    for (int h = 0; h < G; ++h) {
      const float4 s = *reinterpret_cast<const float4*>(scores + h * pitch + j);
      const float z = lse2[h];
      w[0] += __builtin_amdgcn_exp2f(s.x - z);
      w[1] += __builtin_amdgcn_exp2f(s.y - z);
      w[2] += __builtin_amdgcn_exp2f(s.z - z);
      w[3] += __builtin_amdgcn_exp2f(s.w - z);
    }
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      if (j + x < e.n) {
        const float sum = old[x] + w[x];
        acc[j + x] = sum;
        if (may_go(e, j + x)) best = smaller(best, Candidate{sum, j + x});
      } else if (j + x == e.n) {
        *own = w[x];
      }
    }
  }
  return best;
}

// Slot `slot` (-1: none) of `heads` heads from g0 on takes the oldest recent state, that one's place (or the row behind the cache) the
// token's.  own: the token's weights by head.
template <int THREADS>
__device__ inline void move_states(const EvictStep& e, int b, int l, int g0, int heads, int slot, const float* own) {
  const int to = e.oldest >= 0 ? e.oldest : e.n;
  const int esz = e.row_bytes / e.dm.D, pieces = e.row_bytes / 16;
  for (int x = threadIdx.x; x < heads * 2 * pieces; x += THREADS) {
    const int g = g0 + x / (2 * pieces), piece = x % pieces;
    const bool is_v = x / pieces % 2;
    const View &from = is_v ? e.v_new : e.k_new, &cache = is_v ? e.v_cache : e.k_cache;
    char* rows = static_cast<char*>(const_cast<void*>(cache.ptr)) + (b * cache.sb + l * cache.sl + g * cache.sh) * esz;
    const char* src = static_cast<const char*>(from.ptr) + (b * from.sb + l * from.sl + g * from.sh) * esz;
    uint4* at = reinterpret_cast<uint4*>(rows + to * cache.ss * esz) + piece;
    const uint4 fresh = reinterpret_cast<const uint4*>(src)[piece], moved = slot >= 0 ? *at : fresh;
    if (slot >= 0 && slot != to) *(reinterpret_cast<uint4*>(rows + slot * cache.ss * esz) + piece) = moved;
    *at = fresh;
  }
  const int64_t unit0 = static_cast<int64_t>(b * e.dm.L + l) * e.dm.Hkv + g0;
  for (int h = threadIdx.x; h < heads; h += THREADS) {
    float* acc = e.acc + (unit0 + h) * e.acc_pitch;
    if (slot >= 0) acc[slot] = acc[to];
    acc[to] = own[h];
  }
}

// The whole unit.  lse2: by head, in LDS; scratch (LDS): Candidates of the waves and the token's weight behind them.  acc is read by
// threads other than the ones that wrote it, behind a barrier.
template <int THREADS>
__device__ inline void evict_unit(const EvictStep& e, int b, int l, int g, const float* scores, int64_t pitch, const float* lse2,
                                  Candidate* scratch) {
  const int64_t unit = static_cast<int64_t>(b * e.dm.L + l) * e.dm.Hkv + g;
  float* const own = reinterpret_cast<float*>(scratch + THREADS / 64);
  Candidate best = grow_sums<THREADS>(e, scores, pitch, lse2, e.acc + unit * e.acc_pitch, 0, e.n + 1, own);
  best = smallest_of_block<THREADS>(best, scratch);
  const int slot = e.oldest >= 0 ? best.slot : -1;
  move_states<THREADS>(e, b, l, g, 1, slot, own);
  if (threadIdx.x == 0 && e.evicted != nullptr) e.evicted[unit] = slot;
}

}  // namespace
}  // namespace citrus

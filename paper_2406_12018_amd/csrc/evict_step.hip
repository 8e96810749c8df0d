// Eviction by accumulated attention weight, one generated token at a time: behind the attention of the token (its logits and
// normalisers in the workspace), the states' sums grow by the step's weights, and the state with the smallest sum makes room.
//
//   w_j = sum over the heads of the group of exp2(s_j - lse),   sum_j += w_j
#include "few_rows.h"

namespace citrus {
namespace {

constexpr int kThreads = 256;
constexpr int kRangeKeys = 4096;

// The state that goes: the smaller sum, of equal ones the lower slot.  A sum that is not a number is never the smaller one.
struct Candidate {
  float sum;
  int slot;
};
__device__ inline Candidate smaller(const Candidate& a, const Candidate& b) {
  return b.sum < a.sum || (b.sum == a.sum && b.slot < a.slot) ? b : a;
}
__device__ inline Candidate smallest_of_block(Candidate c, Candidate* lds) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) c = smaller(c, Candidate{__shfl_xor(c.sum, o, 64), __shfl_xor(c.slot, o, 64)});
  if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = c;
  __syncthreads();
  c = lds[0];
  for (int w = 1; w < kThreads / 64; ++w) c = smaller(c, lds[w]);
  return c;
}
__device__ inline bool may_go(const EvictStep& a, int slot) {
  return (slot >= a.start && slot < a.n - a.recent) || slot == a.oldest;
}

// grid: (ranges of keys * Hkv, B * L)
__global__ __launch_bounds__(kThreads) void accumulate_kernel(EvictStep a, int ranges, int per_range) {
  __shared__ Candidate lds[kThreads / 64];
  const Dims& dm = a.dm;
  const int g = blockIdx.x / ranges, range = blockIdx.x % ranges;
  const int64_t unit = static_cast<int64_t>(blockIdx.y) * dm.Hkv + g;
  const float* scores = a.scores + unit * dm.G * a.score_pitch;
  const float* lse2 = a.lse2 + unit * dm.G;
  float* acc = a.acc + unit * a.acc_pitch;
  Candidate best{INFINITY, a.oldest};
  const int end = min(a.n + 1, (range + 1) * per_range);
  for (int j = range * per_range + threadIdx.x; j < end; j += kThreads) {
    float w = 0.f;
    for (int h = 0; h < dm.G; ++h) w += exp2f(scores[static_cast<int64_t>(h) * a.score_pitch + j] - lse2[h]);
    if (j == a.n) {
      a.own[unit] = w;
    } else {
      w += acc[j];
      acc[j] = w;
      if (may_go(a, j)) best = smaller(best, Candidate{w, j});
    }
  }
  if (a.oldest < 0) return;
  best = smallest_of_block(best, lds);
  if (threadIdx.x == 0) a.best[unit * ranges + range] = make_float2(best.sum, __int_as_float(best.slot));
}

// One workgroup per selection: the smallest of the ranges' candidates, or of a layer's sums over its heads; then the rows move.
__global__ __launch_bounds__(kThreads) void make_room_kernel(EvictStep a, int ranges, int heads, View kn, View vn, View kc, View vc, int row_bytes) {
  __shared__ Candidate lds[kThreads / 64];
  const Dims& dm = a.dm;
  const int g0 = blockIdx.x * heads;
  const int b = blockIdx.y / dm.L, l = blockIdx.y % dm.L;
  const int64_t unit0 = static_cast<int64_t>(blockIdx.y) * dm.Hkv + g0;
  int slot = -1;
  if (a.oldest >= 0) {
    Candidate best{INFINITY, a.oldest};
    if (heads == 1) {
      for (int r = threadIdx.x; r < ranges; r += kThreads) {
        const float2 c = a.best[unit0 * ranges + r];
        best = smaller(best, Candidate{c.x, __float_as_int(c.y)});
      }
    } else {
      for (int j = threadIdx.x; j < a.n; j += kThreads) {
        if (!may_go(a, j)) continue;
        float sum = 0.f;
        for (int h = 0; h < heads; ++h) sum += a.acc[(unit0 + h) * a.acc_pitch + j];
        best = smaller(best, Candidate{sum, j});
      }
    }
    best = smallest_of_block(best, lds);
    slot = best.slot;
  }
  __syncthreads();
  const int to = a.oldest >= 0 ? a.oldest : a.n;  // where the token's state goes
  const int esz = row_bytes / dm.D, pieces = row_bytes / 16;
  for (int e = threadIdx.x; e < heads * 2 * pieces; e += kThreads) {
    const int g = g0 + e / (2 * pieces), piece = e % pieces;
    const bool is_v = e / pieces % 2;
    const View &from = is_v ? vn : kn, &cache = is_v ? vc : kc;
    char* rows = static_cast<char*>(const_cast<void*>(cache.ptr)) + (b * cache.sb + l * cache.sl + g * cache.sh) * esz;
    const char* src = static_cast<const char*>(from.ptr) + (b * from.sb + l * from.sl + g * from.sh) * esz;
    uint4* at = reinterpret_cast<uint4*>(rows + to * cache.ss * esz) + piece;
    if (slot >= 0 && slot != to) *(reinterpret_cast<uint4*>(rows + slot * cache.ss * esz) + piece) = *at;
    *at = reinterpret_cast<const uint4*>(src)[piece];
  }
  for (int h = threadIdx.x; h < heads; h += kThreads) {
    float* acc = a.acc + (unit0 + h) * a.acc_pitch;
    if (slot >= 0) acc[slot] = acc[to];
    acc[to] = a.own[unit0 + h];
  }
  if (threadIdx.x == 0 && a.evicted != nullptr) a.evicted[static_cast<int64_t>(blockIdx.y) * gridDim.x + blockIdx.x] = slot;
}

}  // namespace

int evict_step_ranges(int n) { return n / kRangeKeys + 1; }  // of the n states and the token's own

hipError_t launch_evict_step(int elem_bytes, const EvictStep& a, bool per_layer, View k_new, View v_new, View k_cache, View v_cache,
                             hipStream_t st) {
  const int per_range = kRangeKeys, ranges = evict_step_ranges(a.n);
  hipLaunchKernelGGL(accumulate_kernel, dim3(ranges * a.dm.Hkv, a.dm.B * a.dm.L), dim3(kThreads), 0, st, a, ranges, per_range);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int heads = per_layer ? a.dm.Hkv : 1;
  hipLaunchKernelGGL(make_room_kernel, dim3(a.dm.Hkv / heads, a.dm.B * a.dm.L), dim3(kThreads), 0, st, a, ranges, heads, k_new, v_new,
                     k_cache, v_cache, a.dm.D * elem_bytes);
  return hipGetLastError();
}

}  // namespace citrus

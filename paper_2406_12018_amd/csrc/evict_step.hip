// Eviction by accumulated attention weight, one generated token at a time, where the launch that attends does not evict itself: its
// logits and its ranges' parts of the rows are in the workspace.
#include "evict_unit.h"

namespace citrus {
namespace {

// The G rows of a unit from their ranges of keys: their log-sum-exp (base 2) to lse2 in LDS, their results to `out` where `store` says so.
template <typename E, int D, int THREADS>
__device__ inline void rows_of_unit(const FewRows& a, int b, int l, int g, bool store, float* lse2) {
  const int G = a.dm.G;
  const int64_t row0 = static_cast<int64_t>(b * a.dm.L + l) * a.dm.Hq + g * G;
  if (store) {
    for (int x = threadIdx.x; x < G * (D / 4); x += THREADS) {
      const int h = x / (D / 4), d = x % (D / 4) * 4;
      RowParts p = join_ranges<D>(a, row0 + h, d);
      finish_row<E>(a, b, l, g * G + h, 0, row0 + h, d, p, true, lse2 + h);
    }
  } else {
    const int64_t all = static_cast<int64_t>(a.dm.B) * a.dm.L * a.dm.Hq;
    for (int h = threadIdx.x; h < G; h += THREADS) {
      RowParts p;
      for (int s = 0; s < a.splits; ++s) p.m = fmaxf(p.m, a.part_ml[s * all + row0 + h].x);
      for (int s = 0; s < a.splits; ++s) p.add(a.part_ml[s * all + row0 + h], make_float4(0.f, 0.f, 0.f, 0.f));
      lse2[h] = p.reference() + log2f(p.sum);
    }
  }
  __syncthreads();
}

// One workgroup per unit.  grid: (Hkv, B * L); LDS: G floats.  At 4096 keys of one layer two launches in ranges take 13 us, this one 9.
constexpr int kUnitThreads = 512, kUnitKeys = 8192;
template <typename E, int D>
__global__ __launch_bounds__(kUnitThreads) void evict_unit_kernel(FewRows a, EvictStep e) {
  extern __shared__ float lse2[];
  __shared__ EvictLds<kUnitThreads> lds;
  const int g = blockIdx.x, b = a.by_layers.quotient(blockIdx.y), l = blockIdx.y - b * a.dm.L;
  EvictAhead<kUnitThreads> ahead;
  ahead.ask(e, b, l, g);
  const float* scores = a.scores + (static_cast<int64_t>(blockIdx.y) * a.dm.Hq + g * a.dm.G) * a.score_pitch;
  const TwoTurns first = first_turns<kUnitThreads>(e, scores, a.score_pitch, 0, e.n + 1);
  rows_of_unit<E, D, kUnitThreads>(a, b, l, g, true, lse2);
  evict_unit<kUnitThreads>(e, b, l, g, scores, a.score_pitch, lse2, ahead, first, lds);
}

// Long caches and selections per layer: the sums grow in ranges of keys, and one workgroup per selection makes room behind them.
constexpr int kThreads = 256;
constexpr int kRangeKeys = 4096;
// grid: (ranges * Hkv, B * L)
template <typename E, int D>
__global__ __launch_bounds__(kThreads) void grow_sums_kernel(FewRows a, EvictStep e, int ranges) {
  extern __shared__ float lse2[];
  __shared__ EvictLds<kThreads> lds;
  const int g = blockIdx.x / ranges, range = blockIdx.x % ranges, b = a.by_layers.quotient(blockIdx.y), l = blockIdx.y - b * a.dm.L;
  const int64_t unit = static_cast<int64_t>(blockIdx.y) * a.dm.Hkv + g;
  float* const acc = e.acc + unit * e.acc_pitch;
  const int begin = range * kRangeKeys, end = min(e.n + 1, begin + kRangeKeys);
  const Sums4 sums = load_sums(e, acc, begin + 4 * threadIdx.x);
  const float* scores = a.scores + unit * a.dm.G * a.score_pitch;
  const TwoTurns first = first_turns<kThreads>(e, scores, a.score_pitch, begin, end);
  rows_of_unit<E, D, kThreads>(a, b, l, g, range == 0, lse2);
  const Candidate mine = grow_sums<kThreads>(e, scores, a.score_pitch, lse2, acc, begin, end, sums, first, lds);
  const Candidate best = smallest_of_block<kThreads>(mine, lds);
  if (threadIdx.x == 0) {
    e.best[unit * ranges + range] = make_float2(best.sum, __int_as_float(best.slot));
    if (end == e.n + 1) e.own[unit] = lds.own;
  }
}
// grid: (Hkv / heads, B * L): the smallest of the ranges' candidates, or of a layer's sums over its heads
__global__ __launch_bounds__(kThreads) void make_room_kernel(EvictStep e, int ranges, int heads) {
  __shared__ EvictLds<kThreads> lds;
  const int g0 = blockIdx.x * heads, b = blockIdx.y / e.dm.L, l = blockIdx.y % e.dm.L;
  const int64_t unit0 = static_cast<int64_t>(blockIdx.y) * e.dm.Hkv + g0;
  int slot = -1;
  if (e.oldest >= 0) {
    Candidate best{INFINITY, e.oldest};
    if (heads == 1) {
      for (int r = threadIdx.x; r < ranges; r += kThreads) {
        const float2 c = e.best[unit0 * ranges + r];
        best = smaller(best, Candidate{c.x, __float_as_int(c.y)});
      }
    } else {
      for (int j = threadIdx.x; j < e.n; j += kThreads) {
        float sum = 0.f;
#pragma unroll 8
        for (int h = 0; h < heads; ++h) sum += e.acc[(unit0 + h) * e.acc_pitch + j];
        if (may_go(e, j)) best = smaller(best, Candidate{sum, j});
      }
    }
    slot = smallest_of_block<kThreads>(best, lds).slot;
  }
  for (int x = threadIdx.x; x < heads * 2 * e.row_bytes / 16; x += kThreads) move_piece(e, moving_piece(e, b, l, g0, x), slot);
  for (int h = threadIdx.x; h < heads; h += kThreads) {
    float* const acc = e.acc + (unit0 + h) * e.acc_pitch;
    move_sum(e, acc, slot, slot >= 0 ? acc[e.oldest] : 0.f, e.own[unit0 + h]);
  }
  if (threadIdx.x == 0 && e.evicted != nullptr) e.evicted[static_cast<int64_t>(blockIdx.y) * gridDim.x + blockIdx.x] = slot;
}

template <typename E, int D>
hipError_t launch(const FewRows& a, const EvictStep& e, bool per_layer, hipStream_t st) {
  const dim3 units(e.dm.Hkv, e.dm.B * e.dm.L);
  const size_t lds = e.dm.G * sizeof(float);
  const int ranges = evict_step_ranges(e.n);
  if (!per_layer && e.n < kUnitKeys) {
    hipLaunchKernelGGL((evict_unit_kernel<E, D>), units, dim3(kUnitThreads), lds, st, a, e);
    return hipGetLastError();
  }
  hipLaunchKernelGGL((grow_sums_kernel<E, D>), dim3(ranges * e.dm.Hkv, units.y), dim3(kThreads), lds, st, a, e, ranges);
  const hipError_t err = hipGetLastError();
  if (err != hipSuccess) return err;
  const int heads = per_layer ? e.dm.Hkv : 1;
  hipLaunchKernelGGL(make_room_kernel, dim3(e.dm.Hkv / heads, units.y), dim3(kThreads), 0, st, e, ranges, heads);
  return hipGetLastError();
}

}  // namespace

int evict_step_ranges(int n) { return n / kRangeKeys + 1; }  // of the n states and the token's own

hipError_t launch_evict_step(int dtype, const FewRows& a, const EvictStep& e, bool per_layer, hipStream_t st) {
  if (dtype == CITRUS_BF16) return e.dm.D == 128 ? launch<uint16_t, 128>(a, e, per_layer, st) : launch<uint16_t, 64>(a, e, per_layer, st);
  return e.dm.D == 128 ? launch<float, 128>(a, e, per_layer, st) : launch<float, 64>(a, e, per_layer, st);
}

}  // namespace citrus

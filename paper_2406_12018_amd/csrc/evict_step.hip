// Eviction by accumulated attention weight, one generated token at a time, where the launch that attends does not evict itself: its
// logits and its ranges' parts of the rows are in the workspace.  It reads G logits and a sum per state and writes the sum: bound by its
// chain of reads where there are few units (8 units of 768 states 7.5 us), by memory where there are many (640 units of 4096 states,
// eight heads each, 28 us = 4.4 TB/s).
#include "evict_unit.h"

namespace citrus {
namespace {

// The rows of `units` KV heads from g on, from their ranges of keys: their log-sum-exp (base 2) to lse2 in LDS, their results to `out` where
// `store` says so.
template <typename E, int D, int THREADS>
__device__ inline void rows_of_units(const FewRows& a, int b, int l, int g, int units, bool store, float* lse2) {
  const int rows = a.dm.G * units;
  const int64_t row0 = static_cast<int64_t>(b * a.dm.L + l) * a.dm.Hq + g * a.dm.G;
  if (store) {
    for (int x = threadIdx.x; x < rows * (D / 4); x += THREADS) {
      const int h = x / (D / 4), d = x % (D / 4) * 4;
      RowParts p = join_ranges<D>(a, row0 + h, d);
      finish_row<E>(a, b, l, g * a.dm.G + h, 0, row0 + h, d, p, true, lse2 + h);
    }
  } else {
    const int64_t all = static_cast<int64_t>(a.dm.B) * a.dm.L * a.dm.Hq;
    for (int h = threadIdx.x; h < rows; h += THREADS) {
      RowParts p;
      for (int s = 0; s < a.splits; ++s) p.m = fmaxf(p.m, a.part_ml[s * all + row0 + h].x);
      for (int s = 0; s < a.splits; ++s) p.add(a.part_ml[s * all + row0 + h], make_float4(0.f, 0.f, 0.f, 0.f));
      lse2[h] = p.reference() + __builtin_amdgcn_logf(p.sum);  // as finish_row forms it
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
  rows_of_units<E, D, kUnitThreads>(a, b, l, g, 1, true, lse2);
  evict_unit<kUnitThreads>(e, b, l, g, scores, a.score_pitch, lse2, ahead, first, lds);
}

// One workgroup per layer, for a selection per layer: a thread has four keys, of all heads one after the other, and the sum of their sums
// in head order.  LDS: Hq + 2 Hkv floats.  grid: (1, B * L).  Two launches
// otherwise: 12 heads over 501 states, f32, 11.3 us and their gap, this one 9.5; with 32 heads over 1024 states it takes 14.5, as the two do.
constexpr int kLayerKeys = 4 * kUnitThreads, kLayerHeads = 16;
template <typename E, int D>
__global__ __launch_bounds__(kUnitThreads) void evict_layer_kernel(FewRows a, EvictStep e) {
  extern __shared__ float lse2[];
  __shared__ EvictLds<kUnitThreads> lds;
  const Dims& dm = a.dm;
  float *const own = lse2 + dm.Hq, *const oldest = own + dm.Hkv;  // by head: the token's weights, the sums of the oldest recent state
  const int b = a.by_layers.quotient(blockIdx.y), l = blockIdx.y - b * dm.L, j = 4 * threadIdx.x, at = min(j, e.n & ~3);
  const int64_t unit0 = static_cast<int64_t>(blockIdx.y) * dm.Hkv;
  const float* const scores = a.scores + unit0 * dm.G * a.score_pitch + at;
  Logits4 logits = load_logits(scores, a.score_pitch, 0, dm.G, 0);
  Sums4 sums = load_sums(e, e.acc + unit0 * e.acc_pitch, j);
  rows_of_units<E, D, kUnitThreads>(a, b, l, 0, dm.Hkv, true, lse2);
  float rank[4] = {0.f, 0.f, 0.f, 0.f};
  for (int g = 0; g < dm.Hkv; ++g) {
    const float* const mine = scores + static_cast<int64_t>(g) * dm.G * a.score_pitch;
    float* const acc = e.acc + (unit0 + g) * e.acc_pitch;
    const int more = g + 1 < dm.Hkv ? 1 : 0;
    const Sums4 old = sums;
    sums = load_sums(e, acc + more * e.acc_pitch, j);
    float w[4] = {0.f, 0.f, 0.f, 0.f};
    for (int h = 0; h < dm.G; h += 4) {
      const Logits4 now = logits;
      logits = h + 4 < dm.G ? load_logits(mine, a.score_pitch, h + 4, dm.G, 0)
                            : load_logits(mine + more * dm.G * a.score_pitch, a.score_pitch, 0, dm.G, 0);
      add_weights(now, lse2 + g * dm.G, h, dm.G, w);
    }
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      if (j + x < e.n) {
        const float sum = old.x[x] + w[x];
        acc[j + x] = sum;
        rank[x] = g == 0 ? sum : rank[x] + sum;
        if (j + x == e.oldest) oldest[g] = sum;
      } else if (j + x == e.n) {
        own[g] = w[x];
      }
    }
  }
  Candidate best{INFINITY, e.oldest};
#pragma unroll
  for (int x = 0; x < 4; ++x)
    if (j + x < e.n && may_go(e, j + x)) best = smaller(best, Candidate{rank[x], j + x});
  best = smallest_of_block<kUnitThreads>(best, lds);
  const int slot = e.oldest >= 0 ? best.slot : -1;
  for (int x = threadIdx.x; x < dm.Hkv * 2 * e.row_bytes / 16; x += kUnitThreads) move_piece(e, moving_piece(e, b, l, 0, x), slot);
  for (int g = threadIdx.x; g < dm.Hkv; g += kUnitThreads) move_sum(e, e.acc + (unit0 + g) * e.acc_pitch, slot, oldest[g], own[g]);
  if (threadIdx.x == 0 && e.evicted != nullptr) e.evicted[blockIdx.y] = slot;
}

// Long caches and other selections per layer: the sums grow in ranges of keys, and one workgroup per selection makes room behind them.
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
  rows_of_units<E, D, kThreads>(a, b, l, g, 1, range == 0, lse2);
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
  if (per_layer && e.n < kLayerKeys && e.dm.Hq <= kLayerHeads) {
    hipLaunchKernelGGL((evict_layer_kernel<E, D>), dim3(1, units.y), dim3(kUnitThreads), (e.dm.Hq + 2 * e.dm.Hkv) * sizeof(float), st, a, e);
    return hipGetLastError();
  }
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

// What the generation kernels share: a few query rows per KV head (the nodes of a drafted tree, one token) over a cache and a
// handful of states of their own.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "bf16_math.h"
#include "citrus_internal.h"

namespace citrus {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

template <typename E>
__device__ inline const E* row_ptr(const View& v, int b, int l, int h, int64_t row) {
  return static_cast<const E*>(v.ptr) + (b * v.sb + l * v.sl + h * v.sh + row * v.ss);
}

__device__ inline void store4(uint16_t* p, const float (&o)[4]) {
  *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3]));
}
__device__ inline void store4(float* p, const float (&o)[4]) { *reinterpret_cast<float4*>(p) = make_float4(o[0], o[1], o[2], o[3]); }

// Parts of a row over different keys become one: what each holds of it is {maximum (base 2), sum} and four elements before the division.
struct RowParts {
  float m = -INFINITY, sum = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
  __device__ float reference() const { return m == -INFINITY ? 0.f : m; }  // nothing seen: every weight is 0
  __device__ void add(const float2& ml, const float4& x) {
    const float w = __builtin_amdgcn_exp2f(ml.x - reference());
    sum = fmaf(ml.y, w, sum);
    o[0] = fmaf(x.x, w, o[0]);
    o[1] = fmaf(x.y, w, o[1]);
    o[2] = fmaf(x.z, w, o[2]);
    o[3] = fmaf(x.w, w, o[3]);
  }
};

// Is there a node t in document b?
__device__ inline bool is_node(const FewRows& a, int b, int t) { return a.words == nullptr || (a.words[b * a.words_sb + t] >> t & 1); }

// Four elements of a row's result, and with the first of them its log-sum-exp.
template <typename E>
__device__ inline void finish_row(const FewRows& a, int b, int l, int h, int t, int64_t row, int d, RowParts& r, bool real, float* lse2 = nullptr) {
  const float inv = 1.f / r.sum;
#pragma unroll
  for (int x = 0; x < 4; ++x) r.o[x] = real ? r.o[x] * inv : 0.f;
  store4(const_cast<E*>(row_ptr<E>(a.out, b, l, h, t)) + d, r.o);
  if (d == 0) {
    const float v = real ? r.reference() + __builtin_amdgcn_logf(r.sum) : -INFINITY;
    if (a.lse != nullptr) a.lse[row] = v * kLn2;
    if (lse2 != nullptr) *lse2 = v;
  }
}

// What the waves of a workgroup leave in LDS for each other: parts of their rows.
struct WaveRow {
  float m, sum;
  int real, spare;
};
// o_s[wave][32 rows][D + 4], rows_s[wave][32]; KH waves share a block of 32 rows.  The workgroup's `here` rows from `first` on of KV head
// g; lse2 (optional, LDS): base 2, by row of this workgroup.
template <typename E, int D, int WAVES, int KH>
__device__ __forceinline__ void join_waves(const FewRows& a, const float* o_s, const WaveRow* rows_s, int b, int l, int g, int first, int here,
                                           int sp, float* lse2 = nullptr) {
  constexpr int kPitch = D + 4, kRowsAtOnce = 64 * WAVES / (D / 4);
  const Dims& dm = a.dm;
  const int nodes = a.ks.c, bl = b * dm.L + l;
  const int d = threadIdx.x % (D / 4) * 4;
#pragma unroll 4
  for (int r = threadIdx.x / (D / 4); r < here; r += kRowsAtOnce) {
    const int at = (r / 32 * KH) * 32 + r % 32;
    RowParts p;
    WaveRow w[KH];
#pragma unroll
    for (int x = 0; x < KH; ++x) w[x] = rows_s[at + 32 * x];
#pragma unroll
    for (int x = 0; x < KH; ++x) p.m = fmaxf(p.m, w[x].m);
#pragma unroll
    for (int x = 0; x < KH; ++x) p.add(make_float2(w[x].m, w[x].sum), *reinterpret_cast<const float4*>(o_s + (at + 32 * x) * kPitch + d));
    const int hq = a.by_nodes.quotient(first + r), t = first + r - hq * nodes, h = g * dm.G + hq;
    const int64_t row = (static_cast<int64_t>(bl) * dm.Hq + h) * nodes + t;
    if (a.part_o == nullptr) {
      finish_row<E>(a, b, l, h, t, row, d, p, w[0].real, lse2 != nullptr ? lse2 + r : nullptr);
    } else {
      const int64_t at_part = static_cast<int64_t>(sp) * dm.B * dm.L * dm.Hq * nodes + row;
      *reinterpret_cast<float4*>(a.part_o + at_part * D + d) = make_float4(p.o[0], p.o[1], p.o[2], p.o[3]);
      if (d == 0) a.part_ml[at_part] = make_float2(p.m, p.sum);
    }
  }
}

// Four elements of a row from its ranges of keys, four ranges' loads in flight at a time.
template <int D>
__device__ inline RowParts join_ranges(const FewRows& a, int64_t row, int d) {
  const int64_t all = static_cast<int64_t>(a.dm.B) * a.dm.L * a.dm.Hq * a.ks.c;
  RowParts p;
  for (int s = 0; s < a.splits; s += 4) {
    float2 ml[4];
    float4 o[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const int64_t at = min(s + x, a.splits - 1) * all + row;
      ml[x] = a.part_ml[at];
      o[x] = *reinterpret_cast<const float4*>(a.part_o + at * D + d);
    }
    const float before = p.m;
#pragma unroll
    for (int x = 0; x < 4; ++x) p.m = fmaxf(p.m, ml[x].x);
    const float w = __builtin_amdgcn_exp2f(before - p.reference());
    p.sum *= w;
#pragma unroll
    for (int x = 0; x < 4; ++x) p.o[x] *= w;
#pragma unroll
    for (int x = 0; x < 4; ++x)
      if (s + x < a.splits) p.add(ml[x], o[x]);
  }
  return p;
}

// Where a workgroup of the attention is.  grid: (row groups * key ranges, Hkv, B * L).  Workgroups go to the eight XCDs in turn, each with an
// L2 of its own: the row groups that read the same keys are eight workgroups apart.  Next to each other, every one of them had
// the keys from memory: seven ragged documents, 61 nodes over up to 4352 states, two row groups, 550 us, now 538.
template <bool GROUPS>  // are there several row groups, maybe?
struct Place {
  int sp, row_group, g, b, l;
  __device__ explicit Place(const FewRows& a) {
    int bl = blockIdx.z;
    sp = blockIdx.x;
    g = blockIdx.y;
    row_group = 0;
    if (GROUPS && a.row_groups > 1) {
      constexpr int kXcds = 8;
      const int w = blockIdx.x + gridDim.x * (blockIdx.y + gridDim.y * blockIdx.z);
      const int eights = a.units / kXcds, eight = a.by_eights.quotient(w);  // eight keys' units and all their row groups
      int unit;
      if (eight < eights) {
        const int r = w - eight * (kXcds * a.row_groups);
        row_group = r / kXcds;
        unit = eight * kXcds + r % kXcds;
      } else {
        const int left = a.units - eights * kXcds, r = w - eights * (kXcds * a.row_groups);
        row_group = r / left;
        unit = eights * kXcds + r % left;
      }
      const int head = a.by_splits.quotient(unit);
      sp = unit - head * a.splits;
      bl = a.by_heads.quotient(head);
      g = head - bl * a.dm.Hkv;
    }
    b = a.by_layers.quotient(bl);
    l = bl - b * a.dm.L;
  }
};

// What a lane sees of 32 keys, the first of them its document's own state `own` (below 0: cached): bit j, by its node's word.
__device__ inline uint32_t seen_keys(uint64_t word, int own) {
  if (own <= -32) return ~0u;
  return own >= 0 ? static_cast<uint32_t>(word >> own) : static_cast<uint32_t>(word) << -own | ((1u << -own) - 1);
}

}  // namespace
}  // namespace citrus

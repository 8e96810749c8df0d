// Attention of a few query rows per KV head in f32, on the f32 matrix instructions (v_mfma_f32_32x32x2_f32: f32 products and sums).
//
// The f32 mode is for tests and small models.  A wave takes 32 rows and 32-key tiles of its own, S^T = K.Q^T and O^T = V^T.P^T, straight
// from global memory: the weights leave the first product in the layout that the second reads, so nothing goes through LDS before
// the waves join.  K of the next tile is on its way during the second product, V during the first.  88 layers of 64/8 heads over 854
// states, one node: head_dim 128 128 us = 4.8 TB/s, head_dim 64 75 us = 4.1 TB/s (two waves a SIMD, 32 columns of a product for 8 rows);
// with 16 nodes, four row groups, 229 us.  Loads marked as not to be kept were slower (each 16-byte piece of a key is a load of its own).
#include "evict_unit.h"

namespace citrus {
namespace {

typedef __attribute__((ext_vector_type(16))) float f32x16;

constexpr int kWaves = 4;
template <int D>
struct Lds {
  static constexpr int kRows = kWaves * 32 * (D + 4) * 4, kJoin = kRows + kWaves * 32 * 16;  // o_s, rows_s
  static constexpr int kBytes = kJoin + 32 * 4 + sizeof(EvictLds<64 * kWaves>);             // lse2
};

// What a tile's V is read as: a lane has kOut consecutive elements of a row.
template <int D>
struct Values {
  static constexpr int kOut = D / 32;
  float x[16][kOut];
};

enum class Logits { kNone, kKept, kEvict };
// grid: (row groups * key ranges, Hkv, B * L)
template <int D, Logits LOGITS>
__global__ __launch_bounds__(64 * kWaves) void few_rows_f32_kernel(FewRows a, EvictStep ev) {
  constexpr int kOut = D / 32, kPieces = D / 8;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const Dims& dm = a.dm;
  const int lane = threadIdx.x % 64, col = lane % 32, grp = lane / 32;
  const int wu = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const Place<LOGITS != Logits::kEvict> place(a);
  const int b = place.b, l = place.l, g = place.g, row_group = place.row_group;
  const int nodes = a.ks.c, rows = dm.G * nodes;
  const int n_c = a.lens != nullptr ? min(max(a.lens[b], 0), a.ks.n_c) : a.ks.n_c;
  const int n = n_c + nodes;
  const int row = row_group * 32 + col, head = a.by_nodes.quotient(min(row, rows - 1)), t = min(row, rows - 1) - head * nodes;
  const int h = g * dm.G + head;
  uint64_t word = a.words != nullptr ? a.words[b * a.words_sb + t] : 1;
  if (nodes < 64) word &= (uint64_t{1} << nodes) - 1;
  const bool real = word >> t & 1;
  const float c2 = dm.scale * kLog2e;

  // Elements 8 i + 4 grp .. + 3 of a row are this lane's part of its products, of a query and of a key alike.
  float4 q[kPieces], k[kPieces];
#pragma unroll
  for (int i = 0; i < kPieces; ++i) q[i] = *reinterpret_cast<const float4*>(row_ptr<float>(a.q, b, l, h, t) + 8 * i + 4 * grp);
  // Row j of the document's states.  (The views' fields are read here, once: chosen per lane, they were loaded again for every row, and a
  // step over 88 layers of 854 states took 208 us.)
  struct Rows {
    const float *cache, *own;
    int64_t ss_cache, ss_own;
  };
  const Rows ks{row_ptr<float>(a.ks.cache, b, l, g, 0), row_ptr<float>(a.ks.chunk, b, l, g, 0), a.ks.cache.ss, a.ks.chunk.ss};
  const Rows vs{row_ptr<float>(a.vs.cache, b, l, g, 0), row_ptr<float>(a.vs.chunk, b, l, g, 0), a.vs.cache.ss, a.vs.chunk.ss};
  auto state = [&](const Rows& r, int j) {  // past the last state: the last
    j = min(j, n - 1);
    return j < n_c ? r.cache + j * r.ss_cache : r.own + (j - n_c) * r.ss_own;
  };
  auto load_keys = [&](int x) {
    const float* p = state(ks, 32 * x + col) + 4 * grp;
#pragma unroll
    for (int i = 0; i < kPieces; ++i) k[i] = *reinterpret_cast<const float4*>(p + 8 * i);
  };

  float m = -INFINITY, sum = 0.f;
  f32x16 o[kOut];
#pragma unroll
  for (int r = 0; r < kOut; ++r)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[r][i] = 0.f;
  float* scores = nullptr;
  if constexpr (LOGITS != Logits::kNone)
    if (row < rows) scores = a.scores + (static_cast<int64_t>(b * dm.L + l) * dm.Hq + h) * a.score_pitch;

  const int tiles = (n + 31) / 32, per = (tiles + a.splits - 1) / a.splits, end = min(tiles, (place.sp + 1) * per);
  const float* const v_lane = vs.cache + 4 * grp * vs.ss_cache + kOut * col;
  int x = place.sp * per + wu;
  const int whole = min(end, n_c / 32);  // tiles of cached states that every row sees
  if (x < end) load_keys(x);
  auto turn = [&]<bool LAST>() {
    const int j0 = 32 * x, own = j0 - n_c;
    Values<D> v;  // of key 8 (i / 4) + 4 grp + i % 4: elements kOut col .. + kOut - 1
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int key = 8 * (i / 4) + i % 4;
      const float* p = LAST ? state(vs, j0 + key + 4 * grp) + kOut * col : v_lane + (j0 + key) * vs.ss_cache;
      if constexpr (kOut == 4) {
        const float4 w = *reinterpret_cast<const float4*>(p);
        v.x[i][0] = w.x, v.x[i][1] = w.y, v.x[i][2] = w.z, v.x[i][3] = w.w;
      } else {
        const float2 w = *reinterpret_cast<const float2*>(p);
        v.x[i][0] = w.x, v.x[i][1] = w.y;
      }
    }
    f32x16 s;
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      s = __builtin_amdgcn_mfma_f32_32x32x2f32(k[i].x, q[i].x, s, 0, 0, 0);
      s = __builtin_amdgcn_mfma_f32_32x32x2f32(k[i].y, q[i].y, s, 0, 0, 0);
      s = __builtin_amdgcn_mfma_f32_32x32x2f32(k[i].z, q[i].z, s, 0, 0, 0);
      s = __builtin_amdgcn_mfma_f32_32x32x2f32(k[i].w, q[i].w, s, 0, 0, 0);
    }
    if (x + kWaves < end) load_keys(x + kWaves);
    const uint32_t seen = LAST ? seen_keys(word, own) : ~0u;
    if constexpr (LAST) {
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (!(seen >> (8 * (i / 4) + 4 * grp + i % 4) & 1)) s[i] = -INFINITY;
    }
    if (scores != nullptr) {
#pragma unroll
      for (int i = 0; i < 16; i += 4)
        *reinterpret_cast<float4*>(scores + j0 + 2 * i + 4 * grp) = make_float4(s[i] * c2, s[i + 1] * c2, s[i + 2] * c2, s[i + 3] * c2);
    }
    float mx = s[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) mx = fmaxf(mx, s[i]);
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
    const float m_new = fmaxf(m, mx * c2), m_use = m_new == -INFINITY ? 0.f : m_new;
    const float alpha = __builtin_amdgcn_exp2f(m - m_use);
    m = m_new;
    sum *= alpha;
    float p[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      p[i] = __builtin_amdgcn_exp2f(fmaf(s[i], c2, -m_use));
      sum += p[i];
    }
#pragma unroll
    for (int r = 0; r < kOut; ++r)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[r][i] *= alpha;
    if constexpr (LAST) {
      // 0 x infinity is NaN: values that are infinite or NaN are taken out, and their products added to the rows that see them
      float zero = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i)
#pragma unroll
        for (int r = 0; r < kOut; ++r) zero = fmaf(v.x[i][r], 0.f, zero);
      if (__any(zero != 0.f)) {
#pragma unroll 1
        for (int key = 0; key < 32; ++key) {
          const int at = 4 * (key / 8) + key % 4;
          float pk = 0.f;
#pragma unroll
          for (int i = 0; i < 16; ++i) pk = at == i ? p[i] : pk;
          pk = __shfl(pk, col + 32 * (key / 4 % 2), 64);
          const float* value = state(vs, j0 + key);
          const bool sees = seen >> key & 1;
#pragma unroll
          for (int r = 0; r < kOut; ++r)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const float w = value[kOut * (8 * (i / 4) + 4 * grp + i % 4) + r];
              if (sees && !(fabsf(w) < INFINITY)) o[r][i] = fmaf(pk, w, o[r][i]);
            }
        }
#pragma unroll
        for (int i = 0; i < 16; ++i)
#pragma unroll
          for (int r = 0; r < kOut; ++r) v.x[i][r] = fabsf(v.x[i][r]) < INFINITY ? v.x[i][r] : 0.f;
      }
    }
#pragma unroll
    for (int i = 0; i < 16; ++i)
#pragma unroll
      for (int r = 0; r < kOut; ++r) o[r] = __builtin_amdgcn_mfma_f32_32x32x2f32(v.x[i][r], p[i], o[r], 0, 0, 0);
    x += kWaves;
  };
  while (x < whole) turn.template operator()<false>();
  while (x < end) turn.template operator()<true>();

  sum += __shfl_xor(sum, 32, 64);
  float* const o_s = reinterpret_cast<float*>(lds);
  WaveRow* const rows_s = reinterpret_cast<WaveRow*>(lds + Lds<D>::kRows);
  if (row < rows) {
    if (grp == 0) rows_s[wu * 32 + col] = WaveRow{m, sum, real, 0};
    float* const at = o_s + (wu * 32 + col) * (D + 4);
#pragma unroll
    for (int i = 0; i < 16; ++i)
#pragma unroll
      for (int r = 0; r < kOut; ++r) at[kOut * (8 * (i / 4) + 4 * grp + i % 4) + r] = o[r][i];
  }
  __syncthreads();
  const int here = min(32, rows - row_group * 32);
  if constexpr (LOGITS == Logits::kEvict) {
    EvictAhead<64 * kWaves> ahead;
    ahead.ask(ev, b, l, g);
    float* const lse2 = reinterpret_cast<float*>(lds + Lds<D>::kJoin);
    join_waves<float, D, kWaves, kWaves>(a, o_s, rows_s, b, l, g, 0, here, place.sp, lse2);
    __syncthreads();
    const float* const unit = a.scores + (static_cast<int64_t>(b * dm.L + l) * dm.Hq + g * dm.G) * a.score_pitch;
    evict_unit<64 * kWaves>(ev, b, l, g, unit, a.score_pitch, lse2, ahead, first_turns<64 * kWaves>(ev, unit, a.score_pitch, 0, ev.n + 1),
                            *reinterpret_cast<EvictLds<64 * kWaves>*>(lse2 + 32));
  } else {
    join_waves<float, D, kWaves, kWaves>(a, o_s, rows_s, b, l, g, row_group * 32, here, place.sp);
  }
}

template <int D, Logits LOGITS>
hipError_t launch(const FewRows& a, const FewRowsPlan& p, const EvictStep& ev, hipStream_t st) {
  static LdsLimit limit;
  const auto kernel = few_rows_f32_kernel<D, LOGITS>;
  const hipError_t e = raise_lds_limit(limit, reinterpret_cast<const void*>(kernel), Lds<D>::kBytes);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(kernel, dim3(p.row_groups * a.splits, a.dm.Hkv, a.dm.B * a.dm.L), dim3(64 * kWaves), Lds<D>::kBytes, st, a, ev);
  return hipGetLastError();
}
template <int D>
hipError_t launch_form(const FewRows& a, const FewRowsPlan& p, const EvictStep* ev, hipStream_t st) {
  if (ev == nullptr) return launch<D, Logits::kNone>(a, p, EvictStep{}, st);
  return p.evicts ? launch<D, Logits::kEvict>(a, p, *ev, st) : launch<D, Logits::kKept>(a, p, EvictStep{}, st);
}

}  // namespace

hipError_t launch_few_rows_f32(const FewRows& a, const FewRowsPlan& p, const EvictStep* ev, hipStream_t st) {
  return a.dm.D == 128 ? launch_form<128>(a, p, ev, st) : launch_form<64>(a, p, ev, st);
}

}  // namespace citrus

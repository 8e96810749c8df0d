// Generation over a retained cache: attention of drafted trees and of single tokens, the commit of an accepted path.
//
//   S[t, j] = scale q_t . k_j,   out_t = sum_j softmax_j(S[t, .]) v_j
// over the states j of the row's document: its first len cache rows, then the draft rows that the node's word names.
#include "bf16_math.h"
#include "few_rows.h"

namespace citrus {
namespace {

__device__ inline void store_piece(uint16_t* p, const Piece<uint16_t>& f) {
  uint4 w;
  w.x = pack_bf16x2(f.x[0], f.x[1]);
  w.y = pack_bf16x2(f.x[2], f.x[3]);
  w.z = pack_bf16x2(f.x[4], f.x[5]);
  w.w = pack_bf16x2(f.x[6], f.x[7]);
  *reinterpret_cast<uint4*>(p) = w;
}
__device__ inline void store_piece(float* p, const Piece<float>& f) {
  *reinterpret_cast<float4*>(p) = make_float4(f.x[0], f.x[1], f.x[2], f.x[3]);
}

// One wave per query row: the lanes that share a state hold a 16-byte piece of its row each, the groups of lanes take the
// states in turn and keep a running (maximum, sum, output) of their own, merged at the end.
template <typename E, int D>
__global__ __launch_bounds__(256) void few_rows_kernel(FewRows a) {
  typedef Piece<E> P;
  constexpr int kPieces = D / P::kN, kGroups = 64 / kPieces;
  const Dims& dm = a.dm;
  const int lane = threadIdx.x % 64, piece = lane % kPieces, group = lane / kPieces;
  const int rows = dm.Hq * a.ks.c;
  const int row = blockIdx.x * 4 + threadIdx.x / 64;
  if (row >= rows) return;
  const int b = blockIdx.y / dm.L, l = blockIdx.y % dm.L, h = row / a.ks.c, t = row % a.ks.c, g = h / dm.G;
  const int n_c = a.lens != nullptr ? min(max(a.lens[b], 0), a.ks.n_c) : a.ks.n_c;
  const uint64_t word = a.words != nullptr ? a.words[b * a.words_sb + t] : 1;
  const bool real = word >> t & 1;
  const int n = real ? n_c + a.ks.c : 0;
  const P q = load_piece(row_ptr<E>(a.q, b, l, h, t) + piece * P::kN);
  float m = -INFINITY, sum = 0.f;
  P acc = {};
  for (int j = group; j < n; j += kGroups) {
    if (j >= n_c && !(word >> (j - n_c) & 1)) continue;
    const bool cached = j < n_c;
    const int64_t r = cached ? j : j - n_c;
    const P k = load_piece(row_ptr<E>(cached ? a.ks.cache : a.ks.chunk, b, l, g, r) + piece * P::kN);
    const P v = load_piece(row_ptr<E>(cached ? a.vs.cache : a.vs.chunk, b, l, g, r) + piece * P::kN);
    float s = 0.f;
#pragma unroll
    for (int x = 0; x < P::kN; ++x) s = fmaf(q.x[x], k.x[x], s);
#pragma unroll
    for (int o = kPieces / 2; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
    s *= dm.scale * kLog2e;
    if (a.scores != nullptr && piece == 0) a.scores[(static_cast<int64_t>(blockIdx.y) * dm.Hq + h) * a.score_pitch + j] = s;
    const float m_new = fmaxf(m, s), safe = m_new == -INFINITY ? 0.f : m_new;
    const float old = exp2f(m - safe), p = exp2f(s - safe);
    sum = fmaf(sum, old, p);
#pragma unroll
    for (int x = 0; x < P::kN; ++x) acc.x[x] = fmaf(acc.x[x], old, p * v.x[x]);
    m = m_new;
  }
#pragma unroll
  for (int o = kPieces; o < 64; o <<= 1) {
    const float m2 = __shfl_xor(m, o, 64), sum2 = __shfl_xor(sum, o, 64);
    const float top = fmaxf(m, m2), safe = top == -INFINITY ? 0.f : top;
    const float e1 = exp2f(m - safe), e2 = exp2f(m2 - safe);
    sum = sum * e1 + sum2 * e2;
#pragma unroll
    for (int x = 0; x < P::kN; ++x) acc.x[x] = acc.x[x] * e1 + __shfl_xor(acc.x[x], o, 64) * e2;
    m = top;
  }
#pragma unroll
  for (int x = 0; x < P::kN; ++x) acc.x[x] = real ? acc.x[x] / sum : 0.f;
  if (group == 0) store_piece(const_cast<E*>(row_ptr<E>(a.out, b, l, h, t)) + piece * P::kN, acc);
  if (lane == 0) {
    const int64_t at = (static_cast<int64_t>(blockIdx.y) * dm.Hq + h) * a.ks.c + t;
    const float lse2 = real ? m + log2f(sum) : -INFINITY;
    if (a.lse != nullptr) a.lse[at] = lse2 * kLn2;
    if (a.lse2 != nullptr) a.lse2[at] = lse2;
  }
}

// The accepted path's rows: row len + i of a document's cache takes draft row path[i], i < accepted.
// One thread per 16-byte piece of a row of K and V.
__global__ __launch_bounds__(256) void tree_commit_kernel(Dims dm, View kd, View vd, View kc, View vc, Commit a, int row_bytes) {
  const int pieces = row_bytes / 16, per_head = 2 * pieces * a.path_len;
  const int b = blockIdx.y / dm.L, l = blockIdx.y % dm.L;
  const int e = blockIdx.x * 256 + threadIdx.x;
  const int len = a.lens != nullptr ? min(max(a.lens[b], 0), a.cache_len) : a.cache_len;
  const int accepted = min(min(max(a.accepted[b], 0), a.path_len), a.capacity - len);
  if (e == 0 && l == 0 && a.new_lens != nullptr) a.new_lens[b] = len + accepted;
  if (e >= per_head * dm.Hkv) return;
  const int g = e / per_head, r = e % per_head;
  const int i = r / (2 * pieces), piece = r % pieces;
  const bool is_v = r / pieces % 2;
  if (i >= accepted) return;
  const int node = a.path[static_cast<int64_t>(b) * a.path_len + i];
  if (node < 0 || node >= a.nodes) return;
  const View &from = is_v ? vd : kd, &to = is_v ? vc : kc;
  const int esz = row_bytes / dm.D;
  const char* src = static_cast<const char*>(from.ptr) + (b * from.sb + l * from.sl + g * from.sh + node * from.ss) * esz;
  char* dst = static_cast<char*>(const_cast<void*>(to.ptr)) + (b * to.sb + l * to.sl + g * to.sh + (len + i) * to.ss) * esz;
  reinterpret_cast<uint4*>(dst)[piece] = reinterpret_cast<const uint4*>(src)[piece];
}

}  // namespace

size_t few_rows_workspace_floats(int dtype, const Dims& dm, int rows) {
  return dtype == CITRUS_BF16 ? few_rows_bf16_workspace_floats(dm, rows) : 0;
}

hipError_t launch_few_rows(int dtype, const FewRows& a, hipStream_t st) {
  if (dtype == CITRUS_BF16) return launch_few_rows_bf16(a, st);
  const dim3 grid((a.dm.Hq * a.ks.c + 3) / 4, a.dm.B * a.dm.L);
  const auto kernel = a.dm.D == 128 ? few_rows_kernel<float, 128> : few_rows_kernel<float, 64>;
  hipLaunchKernelGGL(kernel, grid, dim3(256), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_tree_commit(int elem_bytes, const Dims& dm, View k_draft, View v_draft, View k_cache, View v_cache,
                              const Commit& a, hipStream_t st) {
  const int64_t pieces = static_cast<int64_t>(2) * dm.D * elem_bytes / 16 * a.path_len * dm.Hkv;
  hipLaunchKernelGGL(tree_commit_kernel, dim3(static_cast<unsigned>((pieces + 255) / 256), dm.B * dm.L), dim3(256), 0, st, dm,
                     k_draft, v_draft, k_cache, v_cache, a, dm.D * elem_bytes);
  return hipGetLastError();
}

}  // namespace citrus

// Generation over a retained cache: how the attention of drafted trees and of single tokens is launched, the joining of key ranges, the
// commit of an accepted path.
//
//   S[t, j] = scale q_t . k_j,   out_t = sum_j softmax_j(S[t, .]) v_j
// over the states j of the row's document: its first len cache rows, then the draft rows that the node's word names.
#include "few_rows.h"

#include <utility>

namespace citrus {
namespace {

// One thread per four elements of a row.  grid: (.., B * L)
template <typename E, int D>
__global__ __launch_bounds__(256) void join_ranges_kernel(FewRows a) {
  const Dims& dm = a.dm;
  const int nodes = a.ks.c, e = blockIdx.x * 256 + threadIdx.x;
  if (e >= dm.Hq * nodes * (D / 4)) return;
  const int d = e % (D / 4) * 4, r = e / (D / 4), h = a.by_nodes.quotient(r), t = r - h * nodes;
  const int b = a.by_layers.quotient(blockIdx.y), l = blockIdx.y - b * dm.L;
  const int64_t row = static_cast<int64_t>(blockIdx.y) * dm.Hq * nodes + r;
  const bool real = is_node(a, b, t);
  RowParts p = join_ranges<D>(a, row, d);
  finish_row<E>(a, b, l, h, t, row, d, p, real);
}

// Ranges of keys, at most: one KV head, 4 rows over 16000 states 19.6 us (32: 16.8, 128: 30.7), over 130000 38.2 (48.8, 39.9); four units of
// 160 rows over 60000 66 (86, 66).
constexpr int kMostSplits = 64;
constexpr int kFewKeys = 512;
// Keys of a range, at least: 8 KV heads over 832 states, 32 rows 10.8 us (64: 12.2, 256: 12.4), 96 rows 14.9 (16.2, 15.4), but 424 rows 42.6
// (27.2, 42.6); one KV head, 4 rows over 4000 states 12.7 (18.2, 11.3).
constexpr int kLeastKeys = 128;
// Workgroups of a form that the chip holds.
int64_t slots_of(int dtype, const Dims& dm, const FewRowsPlan& p) {
  if (dm.D == 128) return p.waves == 4 && p.kh == 1 ? 512 : 256;  // LDS; in f32 registers
  return dtype == CITRUS_F32 ? 512 : p.waves == 8 ? 256 : p.kh == 1 ? 768 : 512;  // registers, stages in LDS, tiles in LDS
}

// More than 64 rows, a block of 32 to a wave: four waves and few stages in LDS leave room for two workgroups to a compute unit, at head_dim
// 64 for three; eight waves only for one.  head_dim 64: 16 documents, 16 layers of 8 KV heads, 124 rows over 300 states 97.5 and 60.5 us (four
// waves); 3 documents, 8 KV heads, 427 rows over 14000 states 100 and 87.  head_dim 128: 2560 units of 120 rows over 60, 300, 1200 states 108
// and 76, 173 and 132, 442 and 378; 288 of them over 4000 states 193 and 165; of 424 rows over 60, 300, 500 states 347 and 273, 533 and 486,
// 682 and 650; over 700, 1200, 4000 states (of the last 512 units) 848 and 818, 1284 and 1250, 737 and 733, and of 160 rows over 300 states,
// where half of the second workgroup's waves have no rows, 224 and 206: these stay with eight.  Few units of up to 128 rows keep the shorter chain of eight waves that halve a stage (head_dim 64, 300 states, 13.1 and 14.9).
FewRowsPlan form_of(int dtype, const Dims& dm, int nodes, int keys, bool logits) {
  const int blocks = (dm.G * nodes + 31) / 32;
  FewRowsPlan p{};
  const bool alone = blocks == 1 || logits || dtype == CITRUS_F32;  // a block of 32 rows to a workgroup
  const bool many = static_cast<int64_t>(dm.B) * dm.L * dm.Hkv > 256;
  const bool halves = blocks <= (many ? 2 : 4), fours = dm.D == 64 || (many && (blocks <= 4 || (blocks > 6 && keys <= kFewKeys)));
  p.kh = alone ? 4 : halves ? 2 : 1;
  p.waves = alone || blocks == 2 || (fours && !halves) ? 4 : 8;
  const int per = p.waves / p.kh;
  p.row_groups = (blocks + per - 1) / per;
  return p;
}
int64_t workgroups(const Dims& dm, const FewRowsPlan& p) { return static_cast<int64_t>(dm.B) * dm.L * dm.Hkv * p.row_groups; }
int most_splits(int dtype, const Dims& dm, const FewRowsPlan& p) {
  const int64_t s = 8 * slots_of(dtype, dm, p) / workgroups(dm, p);
  return static_cast<int>(s < 1 ? 1 : s > kMostSplits ? kMostSplits : s);
}

// Ranges of keys, and waves to a unit.  What a launch takes is counted in 32-key tiles of a workgroup's stream (0.6 us): the rounds of the
// chip times a workgroup's share of the keys, six tiles for its start and end, and with several ranges the parts of its rows, written
// and read (a sixteenth of a tile each).  An eviction within the launch is six more; another launch costs eight, one that evicts
// fourteen.  An f32 tile of head_dim 128 is two (8 KV heads over 300 states 19.4 us in one range, 13.9 in two).
// Of units with few keys the start and the end are the most part.  A unit to a single wave (bf16, up to 32 rows) puts as many units on a
// compute unit as their tiles fit its LDS, five at head_dim 128, and their starts and ends overlap.  They share its stream, of which one
// alone reaches half; the last of them leave it idle in part; and a wave alone evicts more slowly the longer the unit is.  2560 units of
// one row, head_dim 128, four waves and one: 30 states 46.9 and 18.4 us, 130 states 77.5 and 43.4, 300 states 94.7 and 80.5, 1000 states
// 208 and 209, 4000 states 750 and 802; with two heads each and the eviction 81.8 and 30.9, 109 and 57.0, 136 and 94.9, 264 and 265, 962
// and 1040.
FewRowsPlan plan_for(int dtype, const Dims& dm, int nodes, int most_keys, bool logits, bool may_evict) {
  FewRowsPlan p = form_of(dtype, dm, nodes, most_keys, logits);
  const int64_t groups = workgroups(dm, p), slots = slots_of(dtype, dm, p);
  const int unit = p.kh == 4 ? 32 : 64, tiles = (most_keys + unit - 1) / unit;
  const int rows = dm.G * nodes < 32 * p.waves / p.kh ? dm.G * nodes : 32 * p.waves / p.kh;
  const int tile = dtype == CITRUS_F32 && dm.D == 128 ? 2 : 1;
  int64_t best = INT64_MAX;
  for (int s = 1; s <= most_splits(dtype, dm, p); ++s) {
    const int per = (tiles + s - 1) / s;
    if (s > 1 && per * unit < kLeastKeys) break;
    if ((tiles + per - 1) / per != s) continue;  // no empty ranges
    const bool evicts = may_evict && s == 1;
    const int64_t rounds = (s * groups + slots - 1) / slots, each = per * unit / 32 * tile + 6 + (evicts ? 6 : 0) + (s > 1 ? rows / 16 : 0);
    const int64_t cost = rounds * each + (evicts ? 0 : logits ? 14 : s > 1 ? 8 : 0);
    if (cost < best) best = cost, p.splits = s;
  }
  if (dtype == CITRUS_BF16 && p.kh == 4 && p.row_groups == 1) {
    const int64_t at_once = 256 * (dm.D == 128 ? 5 : may_evict ? 8 : 10), rounds = (groups + at_once - 1) / at_once;
    const int64_t shares = (groups + slots - 1) / slots, idle = shares < 2 ? 0 : (shares < 5 ? shares : 5) - 2;
    const int64_t streams = (shares < 2 * rounds ? 2 * rounds : shares) * tiles + idle * tiles / 2;
    if (streams + rounds * (6 + (may_evict ? 6 + tiles : 0)) + (logits && !may_evict ? 14 : 0) < best) p.waves = p.kh = 1, p.splits = 1;
  }
  p.evicts = may_evict && p.splits == 1;
  return p;
}

hipError_t launch_main(int dtype, FewRows& a, const FewRowsPlan& p, const EvictStep* ev, hipStream_t st) {
  a.splits = p.splits;
  a.row_groups = p.row_groups;
  a.units = static_cast<int>(workgroups(a.dm, p) / p.row_groups * p.splits);
  a.by_splits = fast_div(p.splits);
  a.by_heads = fast_div(a.dm.Hkv);
  a.by_eights = fast_div(8 * p.row_groups);
  a.by_layers = fast_div(a.dm.L);
  a.by_nodes = fast_div(a.ks.c);
  a.part_o = nullptr;
  if (p.splits > 1 || (ev != nullptr && !p.evicts)) {
    const size_t rows = static_cast<size_t>(p.splits) * a.dm.B * a.dm.L * a.dm.Hq * a.ks.c;
    a.part_o = a.workspace;
    a.part_ml = reinterpret_cast<float2*>(a.workspace + rows * a.dm.D);
  }
  return dtype == CITRUS_BF16 ? launch_few_rows_bf16(a, p, ev, st) : launch_few_rows_f32(a, p, ev, st);
}

// The accepted path's rows: row len + i of a document's cache takes draft row path[i], i < accepted.  A thread has a 16-byte piece of K or
// V of a head and moves it for path_rows rows, four of them in flight: as a thread per piece and row, 16 documents x 32 layers x 32
// heads took 53 us, half of it threads behind the accepted rows; now 41.  grid: (.., B * L, shares of the path)
__global__ __launch_bounds__(256) void tree_commit_kernel(Dims dm, View kd, View vd, View kc, View vc, Commit a, int row_bytes, int path_rows) {
  const int pieces = row_bytes / 16, bits = __builtin_ctz(pieces);  // a power of two
  const int b = a.by_layers.quotient(blockIdx.y), l = blockIdx.y - b * dm.L;
  const int e = blockIdx.x * 256 + threadIdx.x;
  const int len = a.lens != nullptr ? min(max(a.lens[b], 0), a.cache_len) : a.cache_len;
  const int accepted = min(min(max(a.accepted[b], 0), a.path_len), a.capacity - len);
  if (e == 0 && l == 0 && blockIdx.z == 0 && a.new_lens != nullptr) a.new_lens[b] = len + accepted;
  const int g = e >> (bits + 1), piece = e & (pieces - 1);
  if (g >= dm.Hkv) return;
  const bool is_v = e >> bits & 1;
  const View &from = is_v ? vd : kd, &to = is_v ? vc : kc;
  const int esz = row_bytes / dm.D;
  const char* src = static_cast<const char*>(from.ptr) + (b * from.sb + l * from.sl + g * from.sh) * esz + 16 * piece;
  char* dst = static_cast<char*>(const_cast<void*>(to.ptr)) + (b * to.sb + l * to.sl + g * to.sh + len * to.ss) * esz + 16 * piece;
  const int32_t* path = a.path + static_cast<int64_t>(b) * a.path_len;
  const int end = min(accepted, static_cast<int>(blockIdx.z + 1) * path_rows);
  for (int i = blockIdx.z * path_rows; i < end; i += 4) {
    int node[4];
    uint4 row[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) node[x] = path[min(i + x, end - 1)];
#pragma unroll
    for (int x = 0; x < 4; ++x) row[x] = *reinterpret_cast<const uint4*>(src + min(max(node[x], 0), a.nodes - 1) * from.ss * esz);
#pragma unroll
    for (int x = 0; x < 4; ++x)
      if (i + x < end && node[x] >= 0 && node[x] < a.nodes) *reinterpret_cast<uint4*>(dst + (i + x) * to.ss * esz) = row[x];
  }
}

}  // namespace

size_t few_rows_workspace_floats(int dtype, const Dims& dm, int rows) {
  size_t most = 0;
  for (int t = 1; t <= rows; ++t)
    for (const auto& [logits, keys] : {std::pair{false, 0}, {false, kFewKeys + 1}, {true, 0}}) {
      if (logits && t > 1) continue;
      const int s = most_splits(dtype, dm, form_of(dtype, dm, t, keys, logits));
      const size_t f = s == 1 && !logits ? 0 : static_cast<size_t>(s) * dm.B * dm.L * dm.Hq * t * (dm.D + 2);
      if (f > most) most = f;
    }
  return most;
}

hipError_t launch_tree_attn(int dtype, FewRows a, hipStream_t st) {
  const FewRowsPlan p = plan_for(dtype, a.dm, a.ks.c, a.ks.n_c + a.ks.c, false, false);
  const hipError_t e = launch_main(dtype, a, p, nullptr, st);
  if (e != hipSuccess || p.splits == 1) return e;
  const auto join = dtype == CITRUS_BF16 ? (a.dm.D == 128 ? join_ranges_kernel<uint16_t, 128> : join_ranges_kernel<uint16_t, 64>)
                                         : (a.dm.D == 128 ? join_ranges_kernel<float, 128> : join_ranges_kernel<float, 64>);
  const int pieces = a.dm.Hq * a.ks.c * (a.dm.D / 4);
  hipLaunchKernelGGL(join, dim3((pieces + 255) / 256, a.dm.B * a.dm.L), dim3(256), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_decode_evict(int dtype, FewRows a, const EvictStep& ev, bool per_layer, hipStream_t st) {
  const FewRowsPlan p = plan_for(dtype, a.dm, 1, a.ks.n_c + 1, true, !per_layer && a.dm.G <= 32);
  const hipError_t e = launch_main(dtype, a, p, &ev, st);
  return e != hipSuccess || p.evicts ? e : launch_evict_step(dtype, a, ev, per_layer, st);
}

hipError_t launch_tree_commit(int elem_bytes, const Dims& dm, View k_draft, View v_draft, View k_cache, View v_cache,
                              const Commit& a, hipStream_t st) {
  const int64_t pieces = static_cast<int64_t>(2) * dm.D * elem_bytes / 16 * dm.Hkv;
  const int64_t blocks = (pieces + 255) / 256 * dm.B * dm.L;
  // Few workgroups: each a share of the path.  Two to a compute unit keep the memory busy.
  const int path_rows = blocks < 512 ? 4 : (a.path_len + 3) / 4 * 4;
  hipLaunchKernelGGL(tree_commit_kernel,
                     dim3(static_cast<unsigned>((pieces + 255) / 256), dm.B * dm.L, (a.path_len + path_rows - 1) / path_rows), dim3(256), 0,
                     st, dm, k_draft, v_draft, k_cache, v_cache, a, dm.D * elem_bytes, path_rows);
  return hipGetLastError();
}

}  // namespace citrus

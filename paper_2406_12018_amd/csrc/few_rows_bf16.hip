// Attention of a few query rows per KV head in bf16: the nodes of drafted trees, single tokens of documents of different lengths, and
// the tokens of a bounded cache, whose logits are kept.
//
// Every byte of K and V is read once, softmax on the way: running maximum and sum per row, accumulators in registers.  With R rows
// of a head group a byte of K/V meets R flop: up to 128 rows the launch is the stream of K/V bytes, from about 256 on it is the
// matrix pipe's and the vector units'.  Forms of one kernel, by rows:
//   private  up to 32: every wave streams 32-key tiles of its own through LDS, with no barrier between the waves; a unit to four waves,
//            or to one wave where many units have few keys each;
//   shared   more: the waves of a workgroup read the same 64-key stages, four of them in LDS, a block of 32 rows per KH waves (KH = 2, up
//            to 128 rows: each takes half of a stage's keys; KH = 1, four or eight blocks to a workgroup), one barrier a stage.  Four
//            blocks have fewer stages, so that two workgroups share a compute unit, at head_dim 64 three.
// Keys are split over workgroups where the units do not fill the chip; another launch joins the ranges.
// Measured on an MI355X, a call among others, inputs in turn from three sets: 16 ragged documents, 4 layers of 32/32 heads, head_dim 64, single
// tokens over up to 2048 states 106 us = 6.6 TB/s; 13 nodes, 32/8 heads, 2 layers, over 131072 states 176 us = 6.1 TB/s; 24 nodes, 32 layers
// of 32/8 heads over 1280 states 42 us = 4.4 TB/s with a start and an end of about 8; 61 nodes, 7 ragged documents, 8 layers of 64/8 heads
// over up to 4352 states 538 us = 0.51 PFLOP/s without the second words of the weights, matrix pipe busy 46 % of the SIMD cycles, vector
// units 47 %: eight waves a compute unit do not cover each other's waits.  There, two tiles a step, 128-key stages, a wave priority around the products, fewer address instructions, and one wait
// for all of a tile's reads of LDS changed nothing.  A launch of one tile takes 7.7 us: reads that depend on each other, and instructions that no one has fetched yet.
#include "evict_unit.h"
#include "key_stream.h"

namespace citrus {
namespace {

typedef __attribute__((address_space(3))) void* lds_void_ptr;
typedef __attribute__((address_space(3))) char* lds_char_ptr;

constexpr int kStageKeys = 64;  // shared form
template <int D, int WAVES, int KH>
constexpr int kStagesOf = WAVES == 4 && KH == 1 ? (D == 64 ? 3 : 2) : 4;  // three workgroups to a compute unit, two
// A weight is two bf16 words in P.V, the second what the first leaves out of the f32 value: together off by 2^-16 of it at most, which
// is nothing beside the rounding of the result.  With one word the error of a row would be sqrt(2) times that of this rounding, and a
// row's error has to be the same in every form: which of them serves a tree goes by its number of nodes.  Where the stream of keys bounds
// the second word costs nothing; beyond 128 rows half as many products more: 320 units of 424 rows over 60, 300, 1200 states 41 and 44, 62
// and 71, 149 and 183 us.
constexpr int kWeightParts = 2;
constexpr int kLdsOfUnit = 160 * 1024, kLdsOfVote = 1024;  // __syncthreads_and has some of its own, in front of the tiles

// What the lanes of one query row hold of it.
template <int D>
struct Column {
  float m = -INFINITY, l = 0.f;  // running maximum (base 2), this lane's part of the sum
  f32x16 o[Geo<D>::kOut];
};

// Zero, unless one of the words is infinite or NaN: those times zero are NaN.  One instruction per two values.
__device__ inline float zero_if_finite(const Pack8& a, float sum) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
    sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, a.w[i]), __builtin_bit_cast(bf16x2, 0u), sum, false);
  return sum;
}

// vmcnt(LEFT), nothing else
template <int LEFT>
__device__ inline void wait_loads() {
  static_assert(LEFT < 64);
  __builtin_amdgcn_s_waitcnt((LEFT & 15) | 7 << 4 | 15 << 8 | (LEFT >> 4) << 14);
  asm volatile("" ::: "memory");
}

// One 32-key tile.  LAST: keys that not every row sees; bit j of `seen` says that this lane's row sees key j of the tile.
// CAREFUL: see few_rows_kernel.
template <int D, bool LAST, bool CAREFUL>
__device__ __forceinline__ void key_tile(uint32_t k_t, uint32_t v_t, const uint32_t (&k_off)[Geo<D>::kKk], const uint32_t (&v_off)[2 * Geo<D>::kOut],
                                         const bf16x8 (&q_op)[Geo<D>::kKk], float c2, uint32_t seen, Column<D>& c, float* scores) {
  typedef Geo<D> T;
  const int lane = threadIdx.x % 64, col = lane % 32, grp = lane / 32;
  f32x16 s_acc;
#pragma unroll
  for (int i = 0; i < 16; ++i) s_acc[i] = 0.f;
  {
    Pack8 a[T::kKk];
    uint32_t addr[T::kKk];
#pragma unroll
    for (int kk = 0; kk < T::kKk; ++kk) addr[kk] = k_t + k_off[kk];
    lds_read_k_operands(a, addr);
#pragma unroll
    for (int kk = 0; kk < T::kKk; ++kk) s_acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[kk].v, q_op[kk], s_acc, 0, 0, 0);
  }
  if constexpr (LAST) {
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (!(seen >> (8 * (i / 4) + 4 * grp + i % 4) & 1)) s_acc[i] = -INFINITY;
  }
  if (scores != nullptr) {
#pragma unroll
    for (int i4 = 0; i4 < 4; ++i4)
      *reinterpret_cast<float4*>(scores + 8 * i4 + 4 * grp) =
          make_float4(s_acc[4 * i4] * c2, s_acc[4 * i4 + 1] * c2, s_acc[4 * i4 + 2] * c2, s_acc[4 * i4 + 3] * c2);
  }
  float mx = s_acc[0];
#pragma unroll
  for (int i = 1; i < 16; ++i) mx = fmaxf(mx, s_acc[i]);
  if (__any(mx * c2 > c.m + kMaxSlack)) {
    // A row's maximum moves only by more than that, and only by what the row sees: moved along with a neighbour's, it would have its weights
    // rounded otherwise, for keys or queries that are not the row's.
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
    const bool moves = mx * c2 > c.m + kMaxSlack;
    const float alpha = moves ? __builtin_amdgcn_exp2f(c.m - mx * c2) : 1.f;  // 0 on the first tile
    c.m = moves ? mx * c2 : c.m;
    c.l *= alpha;
#pragma unroll
    for (int r = 0; r < T::kOut; ++r)
#pragma unroll
      for (int i = 0; i < 16; ++i) c.o[r][i] *= alpha;
  }
  const float m_use = LAST && c.m == -INFINITY ? 0.f : c.m;  // a row that has not seen a state yet
  float p[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) p[i] = __builtin_amdgcn_exp2f(fmaf(s_acc[i], c2, -m_use));
  uint32_t p_pk[kWeightParts][8];
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    split_bf16x2(p[2 * i], p[2 * i + 1], p_pk[0][i], p_pk[1][i]);
    sum += p[2 * i] + p[2 * i + 1];
  }
  c.l += sum;
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    Pack8 av[T::kOut];
    {
      uint32_t addr[2 * T::kOut];
#pragma unroll
      for (int e = 0; e < 2 * T::kOut; ++e) addr[e] = v_t + 16 * half * T::kRowBytes + v_off[e];
      lds_read_v_operands(av, addr);
    }
    if constexpr (CAREFUL) {
      // Values that are infinite or NaN are taken out of the operands and their products added one by one, to the rows that see
      // them: the other rows get the bits that any finite values would give.
      float zero = 0.f;
#pragma unroll
      for (int r = 0; r < T::kOut; ++r) zero = zero_if_finite(av[r], zero);
      if (__any(zero != 0.f)) {
#pragma unroll 1
        for (int key = 16 * half; key < 16 * half + 16; ++key) {
          const int at = 4 * (key / 8) + key % 4;
          float pk = 0.f;
#pragma unroll
          for (int i = 0; i < 16; ++i) pk = at == i ? p[i] : pk;
          pk = __shfl(pk, col + 32 * (key / 4 % 2), 64);
          const bool sees = !LAST || (seen >> key & 1);
#pragma unroll
          for (int r = 0; r < T::kOut; ++r)
#pragma unroll
            for (int i4 = 0; i4 < 4; ++i4) {
              const int c0 = 8 * i4 + 4 * grp, d = 16 * r + c0 % 16 + D / 2 * (c0 / 16);
              const uint32_t addr = v_t + key * T::kRowBytes + ((d / 8) ^ T::swz(key)) * 16 + d % 8 * 2;
              i32x2 w;
              asm volatile("ds_read_b64 %0, %1\n\ts_waitcnt lgkmcnt(0)" : "=v"(w) : "v"(addr) : "memory");
#pragma unroll
              for (int x = 0; x < 4; ++x) {
                const float v = __uint_as_float(x % 2 ? w[x / 2] & 0xffff0000u : static_cast<uint32_t>(w[x / 2]) << 16);
                if (sees && !(fabsf(v) < INFINITY)) c.o[r][4 * i4 + x] = fmaf(pk, v, c.o[r][4 * i4 + x]);
              }
            }
        }
#pragma unroll
        for (int r = 0; r < T::kOut; ++r)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            uint32_t w = av[r].w[i];
            if ((w & 0x7f80u) == 0x7f80u) w &= 0xffff0000u;
            if ((w & 0x7f800000u) == 0x7f800000u) w &= 0xffffu;
            av[r].w[i] = w;
          }
      }
    }
#pragma unroll
    for (int y = 0; y < kWeightParts; ++y) {
      Pack8 pb;
#pragma unroll
      for (int x = 0; x < 4; ++x) pb.w[x] = p_pk[y][4 * half + x];
#pragma unroll
      for (int r = 0; r < T::kOut; ++r) c.o[r] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(av[r].v, pb.v, c.o[r], 0, 0, 0);
    }
  }
}

template <int D, int WAVES, int KH>
struct Lds {
  static constexpr int kRows = WAVES * 32 * (D + 4) * 4, kJoin = kRows + WAVES * 32 * 16;  // o_s, rows_s
  static constexpr int kAfter = kJoin + 32 * 4 + sizeof(EvictLds<64 * WAVES>);            // lse2
  static constexpr int kTiles = KH == WAVES ? WAVES * Geo<D>::kWaveLdsBytes : kStagesOf<D, WAVES, KH> * (kStageKeys / 32) * 2 * Geo<D>::kTileBytes;
  static constexpr int kBytes = ((kAfter > kTiles ? kAfter : kTiles) + 15) / 16 * 16;  // ... the strip of logits
};
// A unit's logits in LDS: the pitch of a head.  Heads four words apart from the same bank.
__host__ __device__ inline int strip_pitch(int n) { return (n + 1 + 31) / 32 * 32 + 4; }

// Where a single token's logits go: to the workspace, for other kernels; or the unit is one workgroup's, which evicts by them.
enum class Logits { kNone, kKept, kEvict, kEvictInLds };
// A matrix product forms 0 x v too, for values that a row does not see, and p_lo x v for the second part of a weight whose first part
// said it all: an infinite or NaN value then leaves NaN in rows that must be finite, or infinite.  Nothing in the loop looks for such
// values; a workgroup whose results are not all finite goes over its keys once more, carefully.
//
// GROUPS: several row groups read the same keys.  grid: (row groups * key ranges, Hkv, B * L)
template <int D, int WAVES, int KH, Logits LOGITS, bool GROUPS>
__global__ __launch_bounds__(64 * WAVES, KH == 1 ? 2 : 1) void few_rows_kernel(FewRows a, EvictStep ev) {
  typedef Geo<D> T;
  constexpr bool kPrivate = KH == WAVES;
  constexpr int kBlocks = WAVES / KH;  // of 32 rows
  constexpr int kStages = kStagesOf<D, WAVES, KH>;
  constexpr int kTileBytes = T::kTileBytes, kR = T::kRowsPerLoad;
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const Dims& dm = a.dm;
  const int lane = threadIdx.x % 64, col = lane % 32, grp = lane / 32;
  const int wu = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const Place<GROUPS> at(a);
  const int b = at.b, l = at.l, g = at.g, row_group = at.row_group;
  const int nodes = a.ks.c, rows = dm.G * nodes;
  const int n_c = a.lens != nullptr ? min(max(a.lens[b], 0), a.ks.n_c) : a.ks.n_c;
  const int n = n_c + nodes;

  // this lane's row: node t of head h
  const int row = (row_group * kBlocks + wu / KH) * 32 + col;
  const bool idle = (row_group * kBlocks + wu / KH) * 32 >= rows;  // a wave without rows helps to load

  const int k_ss_cache = static_cast<int>(a.ks.cache.ss), k_ss_own = static_cast<int>(a.ks.chunk.ss);
  const int v_ss_cache = static_cast<int>(a.vs.cache.ss), v_ss_own = static_cast<int>(a.vs.chunk.ss);
  auto resource = [&](const View& v, int count, int ss) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(row_ptr<uint16_t>(v, b, l, g, 0)), 0,
                                             count > 0 ? ((count - 1) * ss + D) * 2 : 0, kBufferFlags);
  };
  const __amdgpu_buffer_rsrc_t k_rs_cache = resource(a.ks.cache, n_c, k_ss_cache), k_rs_own = resource(a.ks.chunk, nodes, k_ss_own);
  const __amdgpu_buffer_rsrc_t v_rs_cache = resource(a.vs.cache, n_c, v_ss_cache), v_rs_own = resource(a.vs.chunk, nodes, v_ss_own);
  const int fill_row = lane / T::kSegs, fill_pos = lane % T::kSegs;
  // rows j0 + kR i + (0 .. kR - 1), kR rows from `first` on, to K rows at k_t and V rows at v_t.  Past the last state: the last.
  // What no other workgroup reads is loaded as not to be kept: 32 layers, budget 1024, 34.3 -> 30.6 us.
  constexpr int kCachePolicy = GROUPS ? 0 : 2;  // nt
  auto fill = [&](int j0, int first, int count, char* k_t, char* v_t) {
    const bool in_cache = j0 + kR * (first + count) <= n_c;
#pragma unroll
    for (int i = first; i < first + count; ++i) {
      const int r = kR * i + fill_row;
      const int seg = (fill_pos ^ T::swz(r)) * 16;
      const lds_void_ptr kd = (lds_void_ptr)(k_t + kR * i * T::kRowBytes), vd = (lds_void_ptr)(v_t + kR * i * T::kRowBytes);
      if (in_cache) {
        __builtin_amdgcn_raw_ptr_buffer_load_lds(k_rs_cache, kd, 16, (j0 + r) * k_ss_cache * 2 + seg, 0, 0, kCachePolicy);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(v_rs_cache, vd, 16, (j0 + r) * v_ss_cache * 2 + seg, 0, 0, kCachePolicy);
      } else {  // two predicated loads: a resource chosen per lane would be loaded in a serialising loop
        const int j = min(j0 + r, n - 1);
        if (j < n_c) {
          __builtin_amdgcn_raw_ptr_buffer_load_lds(k_rs_cache, kd, 16, j * k_ss_cache * 2 + seg, 0, 0, 0);
          __builtin_amdgcn_raw_ptr_buffer_load_lds(v_rs_cache, vd, 16, j * v_ss_cache * 2 + seg, 0, 0, 0);
        }
        keep_apart();
        if (j >= n_c) {
          __builtin_amdgcn_raw_ptr_buffer_load_lds(k_rs_own, kd, 16, (j - n_c) * k_ss_own * 2 + seg, 0, 0, 0);
          __builtin_amdgcn_raw_ptr_buffer_load_lds(v_rs_own, vd, 16, (j - n_c) * v_ss_own * 2 + seg, 0, 0, 0);
        }
        keep_apart();
      }
    }
  };
  const uint32_t lds_at = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_char_ptr)lds));

  const float c2 = dm.scale * kLog2e;
  Column<D> c;
  float* scores = nullptr;  // of this lane's row
  if constexpr (LOGITS == Logits::kEvictInLds) {
    if (row < rows) scores = reinterpret_cast<float*>(lds + Lds<D, WAVES, KH>::kBytes) + row * strip_pitch(ev.n);
  } else if constexpr (LOGITS != Logits::kNone) {
    if (row < rows) scores = a.scores + (static_cast<int64_t>(b * dm.L + l) * dm.Hq + g * dm.G + row) * a.score_pitch;  // nodes == 1
  }

  EvictAhead<64 * WAVES> ahead;
  if constexpr (LOGITS == Logits::kEvict || LOGITS == Logits::kEvictInLds) ahead.ask(ev, b, l, g);
  bool real = true;  // is there a node at this lane's row?
  auto over_the_keys = [&]<bool CAREFUL>() {
    int at_lane = lane;
    asm volatile("" : "+v"(at_lane));  // what follows from it is formed anew by the second pass: kept for it, it cost the first registers
    const int at_col = at_lane % 32, at_grp = at_lane / 32;
    const int at_row = min((row_group * kBlocks + wu / KH) * 32 + at_col, rows - 1);
    const int head = a.by_nodes.quotient(at_row), node = at_row - head * nodes;
    uint64_t word = 1;
    // per-lane LDS read offsets inside a tile, swizzle included
    uint32_t k_off[T::kKk], v_off[2 * T::kOut];
#pragma unroll
    for (int kk = 0; kk < T::kKk; ++kk) k_off[kk] = at_col * T::kRowBytes + (((2 * kk + at_grp) ^ T::swz(at_col)) * 16);
    const int s16 = at_lane % 16, q16 = at_lane / 16;
    const int v_cl = (T::kSegs / 2 * (q16 % 2) + (s16 % 4) / 2) ^ T::swz(4 * (q16 / 2) + s16 / 4);
#pragma unroll
    for (int e = 0; e < 2 * T::kOut; ++e) v_off[e] = (4 * (q16 / 2) + s16 / 4) * T::kRowBytes + ((e ^ v_cl) * 16) + 8 * (s16 % 2);

    bf16x8 q_op[T::kKk];
    auto load_queries = [&] {  // while the first keys are on their way; what is asked for later is counted from here
      if (a.words != nullptr) word = a.words[b * a.words_sb + node];
      const uint16_t* qp = row_ptr<uint16_t>(a.q, b, l, g * dm.G + head, node) + 8 * at_grp;
#pragma unroll
      for (int kk = 0; kk < T::kKk; ++kk) {
        Pack8 x;
        x.u = *reinterpret_cast<const uint4*>(qp + 16 * kk);
        q_op[kk] = x.v;
      }
      wait_loads<0>();
      real = word >> node & 1;
      if (nodes < 64) word &= (uint64_t{1} << nodes) - 1;
    };
    c.m = -INFINITY;
    c.l = 0.f;
#pragma unroll
    for (int r = 0; r < T::kOut; ++r)
#pragma unroll
      for (int i = 0; i < 16; ++i) c.o[r][i] = 0.f;
    // Tiles of cached states that every row sees come first.  (Apart from the others, in a loop of their own: where the two met in one
    // loop, the accumulators went from one set of registers to another and back with every tile.)
    auto tile = [&]<bool LAST>(int j0, uint32_t k_t, uint32_t v_t) {
      key_tile<D, LAST, CAREFUL>(k_t, v_t, k_off, v_off, q_op, c2, LAST ? seen_keys(word, j0 - n_c) : 0u, c,
                                        LOGITS != Logits::kNone && scores != nullptr ? scores + j0 : nullptr);
    };
    if constexpr (kPrivate) {
      // key tiles of this workgroup's range, dealt to its waves in turn
      const int tiles = (n + 31) / 32, per = (tiles + a.splits - 1) / a.splits;
      const int end = min(tiles, (at.sp + 1) * per), whole = min(end, n_c / 32);
      char* const mine = lds + wu * T::kWaveLdsBytes;  // [buffer][K | V][tile]
      const uint32_t mine_at = lds_at + wu * T::kWaveLdsBytes;
      auto fill_tile = [&](int x, int buf) {
        char* k_t = mine + buf * 2 * kTileBytes;
        fill(x * 32, 0, 32 / kR, k_t, k_t + kTileBytes);
      };
      int x = at.sp * per + wu, buf = 0;
      if (x < end) fill_tile(x, 0);
      load_queries();
      auto turn = [&]<bool LAST>() {
        // the other buffer was last read in the previous turn, whose reads have all returned
        if (x + WAVES < end) {
          fill_tile(x + WAVES, buf ^ 1);
          wait_loads<T::kLoadsPerTile>();
        } else {
          wait_loads<0>();
        }
        const uint32_t k_t = mine_at + buf * 2 * kTileBytes;
        tile.template operator()<LAST>(x * 32, k_t, k_t + kTileBytes);
        x += WAVES;
        buf ^= 1;
      };
      if constexpr (!CAREFUL)
        while (x < whole) turn.template operator()<false>();
      while (x < end) turn.template operator()<true>();
    } else {
      constexpr int kSub = kStageKeys / 32, kStageBytes = 2 * kSub * kTileBytes, kGroups = kStageKeys / kR / WAVES;
      constexpr int kLoads = 2 * kGroups;  // of a wave and stage, at least (the stage behind the cache's last row takes more)
      static_assert(kGroups >= 1 && kSub % KH == 0);
      const int stages = (n + kStageKeys - 1) / kStageKeys, per = (stages + a.splits - 1) / a.splits;
      const int begin = at.sp * per, end = min(stages, begin + per), whole = min(end, n_c / kStageKeys);
      auto fill_stage = [&](int x) {
        char* k_t = lds + (x - begin) % kStages * kStageBytes;
        fill(x * kStageKeys, wu * kGroups, kGroups, k_t, k_t + kSub * kTileBytes);
      };
      if (begin < end) fill_stage(begin);
      load_queries();
      for (int x = begin + 1; x < min(end, begin + kStages - 1); ++x) fill_stage(x);
      int x = begin;
      auto turn = [&]<bool LAST>() {
        // this wave's loads of the stage have landed; behind the barrier everybody's have, and the stage before has been read
        if (x + kStages - 2 < end)
          wait_loads<kLoads*(kStages - 2)>();
        else
          wait_loads<0>();
        asm volatile("s_barrier" ::: "memory");
        if (x + kStages - 1 < end) fill_stage(x + kStages - 1);
        const uint32_t k_t = lds_at + (x - begin) % kStages * kStageBytes, v_t = k_t + kSub * kTileBytes;
#pragma unroll
        for (int y = 0; y < kSub / KH; ++y) {
          const int sub = KH == 1 ? y : wu % KH;
          const int j0 = x * kStageKeys + 32 * sub;
          if (!idle && (!LAST || j0 < n)) tile.template operator()<LAST>(j0, k_t + sub * kTileBytes, v_t + sub * kTileBytes);
        }
        ++x;
      };
      if constexpr (!CAREFUL)
        while (x < whole) turn.template operator()<false>();
      while (x < end) turn.template operator()<true>();
    }
  };
  over_the_keys.template operator()<false>();
  float zero = 0.f;
#pragma unroll
  for (int r = 0; r < T::kOut; ++r)
#pragma unroll
    for (int i = 0; i < 16; ++i) zero = fmaf(c.o[r][i], 0.f, zero);
  const bool good = zero == 0.f || row >= rows || !real;
  bool all_good;
  if constexpr (WAVES == 1)
    all_good = __all(good);
  else
    all_good = __syncthreads_and(good);
  if (!all_good) over_the_keys.template operator()<true>();

  // ---- the waves of a block of rows join through LDS (the tiles have been read when every wave is here) ----
  constexpr int kPitch = D + 4;
  const float l_row = c.l + __shfl_xor(c.l, 32, 64);
  __syncthreads();
  float* const o_s = reinterpret_cast<float*>(lds);                                       // [wave][32 rows][kPitch]
  WaveRow* const rows_s = reinterpret_cast<WaveRow*>(lds + Lds<D, WAVES, KH>::kRows);  // [wave][32]
  if (row < rows) {
    if (grp == 0) rows_s[wu * 32 + col] = WaveRow{c.m, l_row, real, 0};
#pragma unroll
    for (int r = 0; r < T::kOut; ++r)
#pragma unroll
      for (int i4 = 0; i4 < 4; ++i4) {
        // registers 4 i4 .. + 3 are rows c' = 8 i4 + 4 grp + 0..3 of O^T -> head_dim 16 r + (c' % 16) + D / 2 (c' / 16)
        const int c0 = 8 * i4 + 4 * grp;
        *reinterpret_cast<float4*>(o_s + (wu * 32 + col) * kPitch + 16 * r + c0 % 16 + D / 2 * (c0 / 16)) =
            make_float4(c.o[r][4 * i4], c.o[r][4 * i4 + 1], c.o[r][4 * i4 + 2], c.o[r][4 * i4 + 3]);
      }
  }
  __syncthreads();
  const int first = row_group * kBlocks * 32, here = min(kBlocks * 32, rows - first);
  if constexpr (LOGITS == Logits::kNone || LOGITS == Logits::kKept) {
    join_waves<uint16_t, D, WAVES, KH>(a, o_s, rows_s, b, l, g, first, here, at.sp);
  } else {
    float* const lse2 = reinterpret_cast<float*>(lds + Lds<D, WAVES, KH>::kJoin);
    join_waves<uint16_t, D, WAVES, KH>(a, o_s, rows_s, b, l, g, first, here, at.sp, lse2);
    __syncthreads();
    EvictLds<64 * WAVES>& scratch = *reinterpret_cast<EvictLds<64 * WAVES>*>(lse2 + 32);
    const bool in_lds = LOGITS == Logits::kEvictInLds;
    const float* const unit = in_lds ? reinterpret_cast<const float*>(lds + Lds<D, WAVES, KH>::kBytes)
                                     : a.scores + (static_cast<int64_t>(b * dm.L + l) * dm.Hq + g * dm.G) * a.score_pitch;
    const int64_t pitch = in_lds ? strip_pitch(ev.n) : a.score_pitch;
    evict_unit<64 * WAVES>(ev, b, l, g, unit, pitch, lse2, ahead, first_turns<64 * WAVES>(ev, unit, pitch, 0, ev.n + 1), scratch);
  }
}

template <int D, int WAVES, int KH, Logits LOGITS, bool GROUPS = false>
hipError_t launch(const FewRows& a, const EvictStep& ev, int row_groups, hipStream_t st) {
  typedef Lds<D, WAVES, KH> L;
  const int strip = LOGITS == Logits::kEvictInLds ? a.dm.G * strip_pitch(ev.n) * 4 : 0;
  static LdsLimit limit;
  const auto kernel = few_rows_kernel<D, WAVES, KH, LOGITS, GROUPS>;
  const hipError_t e = raise_lds_limit(limit, reinterpret_cast<const void*>(kernel), LOGITS == Logits::kEvictInLds ? kLdsOfUnit - kLdsOfVote : L::kBytes);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(kernel, dim3(row_groups * a.splits, a.dm.Hkv, a.dm.B * a.dm.L), dim3(64 * WAVES), L::kBytes + strip, st, a, ev);
  return hipGetLastError();
}
template <int D>
hipError_t launch_form(const FewRows& a, const FewRowsPlan& p, const EvictStep* ev, hipStream_t st) {
  const EvictStep none{};
  if (p.waves == 1)  // a unit to a wave; its logits, if any, in the workspace: a strip of them in LDS costs waves
    return ev == nullptr ? launch<D, 1, 1, Logits::kNone>(a, none, 1, st)
           : p.evicts    ? launch<D, 1, 1, Logits::kEvict>(a, *ev, 1, st)
                         : launch<D, 1, 1, Logits::kKept>(a, none, 1, st);
  if (ev != nullptr) {
    // the strip lies in LDS where that leaves as many workgroups to a compute unit as there are without it
    const int units = D == 128 ? 1 : 2;
    const bool fits = a.dm.G * strip_pitch(ev->n) * 4 + Lds<D, 4, 4>::kBytes <= kLdsOfUnit / units - kLdsOfVote;
    if (!p.evicts)
      return p.row_groups > 1 ? launch<D, 4, 4, Logits::kKept, true>(a, none, p.row_groups, st)
                              : launch<D, 4, 4, Logits::kKept>(a, none, 1, st);
    return fits ? launch<D, 4, 4, Logits::kEvictInLds>(a, *ev, 1, st) : launch<D, 4, 4, Logits::kEvict>(a, *ev, 1, st);
  }
  if (p.kh == 4) return launch<D, 4, 4, Logits::kNone>(a, none, 1, st);
  if (p.kh == 2) return p.waves == 4 ? launch<D, 4, 2, Logits::kNone>(a, none, 1, st) : launch<D, 8, 2, Logits::kNone>(a, none, 1, st);
  if constexpr (D == 128)
    if (p.waves == 8)
      return p.row_groups > 1 ? launch<D, 8, 1, Logits::kNone, true>(a, none, p.row_groups, st)
                              : launch<D, 8, 1, Logits::kNone>(a, none, 1, st);
  return p.row_groups > 1 ? launch<D, 4, 1, Logits::kNone, true>(a, none, p.row_groups, st)
                          : launch<D, 4, 1, Logits::kNone>(a, none, 1, st);
}

}  // namespace

hipError_t launch_few_rows_bf16(const FewRows& a, const FewRowsPlan& p, const EvictStep* ev, hipStream_t st) {
  return a.dm.D == 128 ? launch_form<128>(a, p, ev, st) : launch_form<64>(a, p, ev, st);
}

}  // namespace citrus

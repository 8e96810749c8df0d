// Eviction by accumulated attention weight, of one unit by one workgroup: for the kernels that stream the unit's keys, and for one behind
// them.
//
//   w_j = sum over the heads of the group of exp2(s_j - lse),   sum_j += w_j
// and the state with the smallest sum makes room for the token's.  Everything that is read is asked for before it is needed: what this
// costs behind a stream of keys is the exchange between the waves.
#pragma once

#include "few_rows.h"
#include "lanes.h"

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
template <int F>
__device__ inline Candidate smaller_by_lane(const Candidate& c) {
  return smaller(c, Candidate{from_lane<F>(c.sum), __float_as_int(from_lane<F>(__int_as_float(c.slot)))});
}
__device__ inline Candidate smallest_of_wave(Candidate c) {
  c = smaller_by_lane<kXor1>(c);
  c = smaller_by_lane<kXor2>(c);
  c = smaller_by_lane<kXor7>(c);  // l ^ 4 holds what l ^ 7 does
  c = smaller_by_lane<kXor8>(c);
  float s0, s1, j0, j1;
  both_of_rows(c.sum, s0, s1);
  both_of_rows(__int_as_float(c.slot), j0, j1);
  c = smaller(Candidate{s0, __float_as_int(j0)}, Candidate{s1, __float_as_int(j1)});
  both_of_halves(c.sum, s0, s1);
  both_of_halves(__int_as_float(c.slot), j0, j1);
  return smaller(Candidate{s0, __float_as_int(j0)}, Candidate{s1, __float_as_int(j1)});
}
__device__ inline bool may_go(const EvictStep& e, int slot) {
  return (slot >= e.start && slot < e.n - e.recent) || slot == e.oldest;
}

// LDS of a workgroup that evicts.
template <int THREADS>
struct EvictLds {
  Candidate best[THREADS / 64];
  float own, oldest;  // the token's weight, the sum of the oldest recent state
};
// the workgroup is in step on return
template <int THREADS>
__device__ inline Candidate smallest_of_block(Candidate c, EvictLds<THREADS>& lds) {
  c = smallest_of_wave(c);
  if (threadIdx.x % 64 == 0) lds.best[threadIdx.x / 64] = c;
  __syncthreads();
  c = lds.best[0];
#pragma unroll
  for (int w = 1; w < THREADS / 64; ++w) c = smaller(c, lds.best[w]);
  return c;
}

struct Sums4 {
  float x[4];
};
__device__ inline Sums4 load_sums(const EvictStep& e, const float* acc, int j) {
  Sums4 s;
#pragma unroll
  for (int x = 0; x < 4; ++x) s.x[x] = acc[max(min(j + x, e.n - 1), 0)];
  return s;
}
// Logits of four keys and four heads from `h` on.
struct Logits4 {
  float4 s[4];
};
__device__ inline Logits4 load_logits(const float* scores, int64_t pitch, int h, int G, int j) {
  Logits4 l;
#pragma unroll
  for (int x = 0; x < 4; ++x) l.s[x] = *reinterpret_cast<const float4*>(scores + min(h + x, G - 1) * pitch + j);
  return l;
}
// w += their weights.  lse2: by head, in LDS.
__device__ inline void add_weights(const Logits4& l, const float* lse2, int h, int G, float (&w)[4]) {
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    const float z = h + x < G ? lse2[h + x] : INFINITY;
    w[0] += __builtin_amdgcn_exp2f(l.s[x].x - z);
    w[1] += __builtin_amdgcn_exp2f(l.s[x].y - z);
    w[2] += __builtin_amdgcn_exp2f(l.s[x].z - z);
    w[3] += __builtin_amdgcn_exp2f(l.s[x].w - z);
  }
}
// Sums of the keys [begin, end) of a unit grow, four keys and four heads a thread and turn, the logits two turns ahead; begin is a multiple
// of 4.  scores: [head][pitch], lse2: by head.  old, first, second: load_sums of the thread's first keys, the logits of its first turns.
// Returns this thread's smallest.
struct Turn {
  int j, h;
  template <int THREADS>
  __device__ Turn next(int G) const { return h + 4 < G ? Turn{j, h + 4} : Turn{j + 4 * THREADS, 0}; }
  __device__ Logits4 logits(const float* scores, int64_t pitch, int G, int end) const {
    return load_logits(scores, pitch, h, G, min(j, (end - 1) & ~3));
  }
};
struct TwoTurns {
  Logits4 first, second;
};
template <int THREADS>
__device__ inline TwoTurns first_turns(const EvictStep& e, const float* scores, int64_t pitch, int begin, int end) {
  const Turn t{begin + 4 * static_cast<int>(threadIdx.x), 0};
  return TwoTurns{t.logits(scores, pitch, e.dm.G, end), t.next<THREADS>(e.dm.G).logits(scores, pitch, e.dm.G, end)};
}
template <int THREADS>
__device__ inline Candidate grow_sums(const EvictStep& e, const float* scores, int64_t pitch, const float* lse2, float* acc, int begin, int end,
                                      Sums4 old, TwoTurns ahead, EvictLds<THREADS>& lds) {
  const int G = e.dm.G;
  Candidate best{INFINITY, e.oldest};
  Sums4 next;
  float w[4];
  for (Turn t{begin + 4 * static_cast<int>(threadIdx.x), 0}; t.j < end; t = t.next<THREADS>(G)) {
    const Logits4 l = ahead.first;
    ahead.first = ahead.second;
    ahead.second = t.next<THREADS>(G).template next<THREADS>(G).logits(scores, pitch, G, end);
    if (t.h == 0) {
      next = load_sums(e, acc, t.j + 4 * THREADS);
#pragma unroll
      for (int x = 0; x < 4; ++x) w[x] = 0.f;
    }
    add_weights(l, lse2, t.h, G, w);
    if (t.h + 4 < G) continue;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      if (t.j + x < e.n) {
        const float sum = old.x[x] + w[x];
        acc[t.j + x] = sum;
        if (may_go(e, t.j + x)) best = smaller(best, Candidate{sum, t.j + x});
        if (t.j + x == e.oldest) lds.oldest = sum;
      } else if (t.j + x == e.n) {
        lds.own = w[x];
      }
    }
    old = next;
  }
  return best;
}

// A 16-byte piece of what moves: of the oldest recent state, and of the token's.
struct MovingPiece {
  uint4 *from, fresh, moved;
  char* rows;  // the piece of row 0
  int64_t pitch;
};
// x: head * 2 * pieces of a row + (K or V) * pieces + piece
__device__ inline MovingPiece moving_piece(const EvictStep& e, int b, int l, int g0, int x) {
  const int esz = e.row_bytes / e.dm.D, pieces = e.row_bytes / 16;  // powers of two
  const int bits = __builtin_ctz(pieces), g = g0 + (x >> (bits + 1)), piece = x & (pieces - 1);
  const bool is_v = x >> bits & 1;
  const View &from = is_v ? e.v_new : e.k_new, &cache = is_v ? e.v_cache : e.k_cache;
  MovingPiece p;
  p.rows = static_cast<char*>(const_cast<void*>(cache.ptr)) + (b * cache.sb + l * cache.sl + g * cache.sh) * esz + 16 * piece;
  p.pitch = cache.ss * esz;
  const char* src = static_cast<const char*>(from.ptr) + (b * from.sb + l * from.sl + g * from.sh) * esz + 16 * piece;
  p.from = reinterpret_cast<uint4*>(p.rows + (e.oldest >= 0 ? e.oldest : e.n) * p.pitch);
  p.fresh = *reinterpret_cast<const uint4*>(src);
  p.moved = e.oldest >= 0 ? *p.from : p.fresh;
  return p;
}
__device__ inline void move_piece(const EvictStep& e, const MovingPiece& p, int slot) {
  if (slot >= 0 && slot != e.oldest) *reinterpret_cast<uint4*>(p.rows + slot * p.pitch) = p.moved;
  *p.from = p.fresh;
}
// ... and of the sums
__device__ inline void move_sum(const EvictStep& e, float* acc, int slot, float oldest, float own) {
  if (slot >= 0) acc[slot] = oldest;
  acc[e.oldest >= 0 ? e.oldest : e.n] = own;
}

// The whole unit, by THREADS threads (at least the pieces of a K and a V row).  Asked for ahead: its first sums and what moves.
template <int THREADS>
struct EvictAhead {
  Sums4 sums;
  MovingPiece piece;
  __device__ void ask(const EvictStep& e, int b, int l, int g) {
    sums = load_sums(e, e.acc + (static_cast<int64_t>(b * e.dm.L + l) * e.dm.Hkv + g) * e.acc_pitch, 4 * threadIdx.x);
    if (threadIdx.x < 2 * e.row_bytes / 16) piece = moving_piece(e, b, l, g, threadIdx.x);
  }
};
template <int THREADS>
__device__ inline void evict_unit(const EvictStep& e, int b, int l, int g, const float* scores, int64_t pitch, const float* lse2,
                                  const EvictAhead<THREADS>& ahead, const TwoTurns& first, EvictLds<THREADS>& lds) {
  const int64_t unit = static_cast<int64_t>(b * e.dm.L + l) * e.dm.Hkv + g;
  float* const acc = e.acc + unit * e.acc_pitch;
  Candidate best = grow_sums<THREADS>(e, scores, pitch, lse2, acc, 0, e.n + 1, ahead.sums, first, lds);
  best = smallest_of_block<THREADS>(best, lds);
  const int slot = e.oldest >= 0 ? best.slot : -1;
  if (threadIdx.x < 2 * e.row_bytes / 16) move_piece(e, ahead.piece, slot);
  if (threadIdx.x == 0) {
    move_sum(e, acc, slot, lds.oldest, lds.own);
    if (e.evicted != nullptr) e.evicted[unit] = slot;
  }
}

}  // namespace
}  // namespace citrus

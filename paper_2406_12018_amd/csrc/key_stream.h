// Streams of K/V tiles through LDS: what the kernels of a few query rows share (one token, the nodes of a drafted tree).
// A wave reads 32-key tiles from LDS as operands of v_mfma_f32_32x32x16_bf16: S^T = K.Q^T, O^T = V^T.P^T, a query row per lane.
#pragma once

#include "bf16_math.h"
#include "few_rows.h"

namespace citrus {
namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) short i16x4;

constexpr int kTileKeys = 32;             // keys per wave tile = rows of one MFMA
constexpr int kBufferFlags = 0x00020000;  // raw buffer resource word 3 on CDNA: 32-bit data format, no swizzle
constexpr float kMaxSlack = 8.0f;

// Tile geometry of one head dimension; the swizzle of a row's 16-byte segments is the chunk-attention kernels'.
template <int D>
struct Geo {
  static constexpr int kSegs = D / 8;
  static constexpr int kRowBytes = 2 * D;                    // unpadded, XOR-swizzled rows
  static constexpr int kTileBytes = kTileKeys * kRowBytes;   // 8 KB of K, the same of V (head_dim 64: 4 KB)
  static constexpr int kWaveLdsBytes = 4 * kTileBytes;       // {K, V} x two buffers
  static constexpr int kRowsPerLoad = 1024 / kRowBytes;
  static constexpr int kLoadsPerTile = 2 * kTileKeys / kRowsPerLoad;  // 16 (8) instructions of 1 KB
  static constexpr int kKk = D / 16, kOut = D / 32;
  static constexpr int kParts = D == 64 ? 2 : 1;  // bf16 parts of a probability in P.V, as in the chunk-attention kernels
  __device__ static constexpr int swz(int row) {
    return D == 128 ? (2 * (row % 8)) ^ ((row / 8) % 2) : (2 * ((row / 2) % 4)) ^ ((row / 8) % 2) ^ (4 * (row % 2));
  }
};

union Pack8 {
  bf16x8 v;
  uint4 u;
  uint32_t w[4];
  i16x4 h[2];
};

__device__ inline const uint16_t* unit_ptr(const View& v, int b, int l, int h) {
  return static_cast<const uint16_t*>(v.ptr) + (b * v.sb + l * v.sl + h * v.sh);
}

typedef __attribute__((ext_vector_type(4))) int i32x4;
typedef __attribute__((ext_vector_type(2))) int i32x2;

// LDS reads of a tile, written as asm: the compiler drains the vector-memory counter in front of every
// LDS read it can see while LDS-direct loads are in flight (it cannot tell that they fill the OTHER
// buffer), which would make each wave wait for the tile it has just requested.  Each block waits for
// its own reads, so nothing the compiler does not know about is left pending.
// The eight 16-byte A operands (32 keys x 16 head_dim values each) of S^T = K.Q^T:
__device__ inline void lds_read_k_operands(Pack8 (&a)[8], const uint32_t (&addr)[8]) {
  i32x4 r0, r1, r2, r3, r4, r5, r6, r7;
  asm volatile(
      "ds_read_b128 %0, %8\n\t"
      "ds_read_b128 %1, %9\n\t"
      "ds_read_b128 %2, %10\n\t"
      "ds_read_b128 %3, %11\n\t"
      "ds_read_b128 %4, %12\n\t"
      "ds_read_b128 %5, %13\n\t"
      "ds_read_b128 %6, %14\n\t"
      "ds_read_b128 %7, %15\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(r0), "=&v"(r1), "=&v"(r2), "=&v"(r3), "=&v"(r4), "=&v"(r5), "=&v"(r6), "=&v"(r7)
      : "v"(addr[0]), "v"(addr[1]), "v"(addr[2]), "v"(addr[3]), "v"(addr[4]), "v"(addr[5]), "v"(addr[6]), "v"(addr[7])
      : "memory");
  a[0].v = __builtin_bit_cast(bf16x8, r0); a[1].v = __builtin_bit_cast(bf16x8, r1);
  a[2].v = __builtin_bit_cast(bf16x8, r2); a[3].v = __builtin_bit_cast(bf16x8, r3);
  a[4].v = __builtin_bit_cast(bf16x8, r4); a[5].v = __builtin_bit_cast(bf16x8, r5);
  a[6].v = __builtin_bit_cast(bf16x8, r6); a[7].v = __builtin_bit_cast(bf16x8, r7);
}
// The four A operands of one 16-key contraction step of O^T = V^T.P^T through transpose reads
// (ds_read_b64_tr_b16; lane mapping as in the chunk-attention kernels): operand r = head_dim tile r,
// read rd = keys 8 rd .. +7 of the step, which lie 8 rows = 2048 bytes further on.
__device__ inline void lds_read_v_operands(Pack8 (&a)[4], const uint32_t (&addr)[8]) {
  i32x2 r0, r1, r2, r3, r4, r5, r6, r7;
  asm volatile(
      "ds_read_b64_tr_b16 %0, %8\n\t"
      "ds_read_b64_tr_b16 %1, %9 offset:2048\n\t"
      "ds_read_b64_tr_b16 %2, %10\n\t"
      "ds_read_b64_tr_b16 %3, %11 offset:2048\n\t"
      "ds_read_b64_tr_b16 %4, %12\n\t"
      "ds_read_b64_tr_b16 %5, %13 offset:2048\n\t"
      "ds_read_b64_tr_b16 %6, %14\n\t"
      "ds_read_b64_tr_b16 %7, %15 offset:2048\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(r0), "=&v"(r1), "=&v"(r2), "=&v"(r3), "=&v"(r4), "=&v"(r5), "=&v"(r6), "=&v"(r7)
      : "v"(addr[0]), "v"(addr[1]), "v"(addr[2]), "v"(addr[3]), "v"(addr[4]), "v"(addr[5]), "v"(addr[6]), "v"(addr[7])
      : "memory");
  a[0].h[0] = __builtin_bit_cast(i16x4, r0); a[0].h[1] = __builtin_bit_cast(i16x4, r1);
  a[1].h[0] = __builtin_bit_cast(i16x4, r2); a[1].h[1] = __builtin_bit_cast(i16x4, r3);
  a[2].h[0] = __builtin_bit_cast(i16x4, r4); a[2].h[1] = __builtin_bit_cast(i16x4, r5);
  a[3].h[0] = __builtin_bit_cast(i16x4, r6); a[3].h[1] = __builtin_bit_cast(i16x4, r7);
}

// head_dim 64: four K operands; two V operands, whose second read lies 8 rows = 1024 bytes further on
__device__ inline void lds_read_k_operands(Pack8 (&a)[4], const uint32_t (&addr)[4]) {
  i32x4 r0, r1, r2, r3;
  asm volatile(
      "ds_read_b128 %0, %4\n\t"
      "ds_read_b128 %1, %5\n\t"
      "ds_read_b128 %2, %6\n\t"
      "ds_read_b128 %3, %7\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(r0), "=&v"(r1), "=&v"(r2), "=&v"(r3)
      : "v"(addr[0]), "v"(addr[1]), "v"(addr[2]), "v"(addr[3])
      : "memory");
  a[0].v = __builtin_bit_cast(bf16x8, r0); a[1].v = __builtin_bit_cast(bf16x8, r1);
  a[2].v = __builtin_bit_cast(bf16x8, r2); a[3].v = __builtin_bit_cast(bf16x8, r3);
}
__device__ inline void lds_read_v_operands(Pack8 (&a)[2], const uint32_t (&addr)[4]) {
  i32x2 r0, r1, r2, r3;
  asm volatile(
      "ds_read_b64_tr_b16 %0, %4\n\t"
      "ds_read_b64_tr_b16 %1, %5 offset:1024\n\t"
      "ds_read_b64_tr_b16 %2, %6\n\t"
      "ds_read_b64_tr_b16 %3, %7 offset:1024\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(r0), "=&v"(r1), "=&v"(r2), "=&v"(r3)
      : "v"(addr[0]), "v"(addr[1]), "v"(addr[2]), "v"(addr[3])
      : "memory");
  a[0].h[0] = __builtin_bit_cast(i16x4, r0); a[0].h[1] = __builtin_bit_cast(i16x4, r1);
  a[1].h[0] = __builtin_bit_cast(i16x4, r2); a[1].h[1] = __builtin_bit_cast(i16x4, r3);
}

// The tile whose loads were issued before the newest kLoadsPerTile ones has landed in LDS.  LDS-direct
// loads complete in order and are counted by the issuing wave's vector-memory counter.  The waits are
// the compiler's own builtin, so that its counter bookkeeping knows about them (a wait hidden in an asm
// statement leaves it believing that the query loads are still pending, and it then drains the counter
// in front of the first LDS read of every iteration, prefetched tile included); the empty asm with a
// memory clobber keeps the LDS reads of the tile behind the wait.
// s_waitcnt immediate on gfx9: vmcnt[3:0] = bits 3:0, expcnt = bits 6:4, lgkmcnt = bits 11:8, vmcnt[5:4] = bits 15:14.
template <int LOADS>
__device__ inline void wait_all_but_newest_tile() {
  static_assert(LOADS == 8 || LOADS == 16, "vmcnt of one tile's load instructions");
  __builtin_amdgcn_s_waitcnt(LOADS == 16 ? 0x4F70 : 0x0F78);  // vmcnt(LOADS), nothing else
  asm volatile("" ::: "memory");
}
__device__ inline void wait_all_loads() {
  __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0), nothing else
  asm volatile("" ::: "memory");
}
// keeps two predicated regions from being merged into one with per-lane operands
__device__ inline void keep_apart() { asm volatile("" ::: "memory"); }

}  // namespace
}  // namespace citrus

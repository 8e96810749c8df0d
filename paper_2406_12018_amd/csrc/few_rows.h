// What the generation kernels share: a few query rows per KV head (the nodes of a drafted tree, one token) over a cache and a
// handful of states of their own.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "citrus_internal.h"

namespace citrus {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

template <typename E>
__device__ inline const E* row_ptr(const View& v, int b, int l, int h, int64_t row) {
  return static_cast<const E*>(v.ptr) + (b * v.sb + l * v.sl + h * v.sh + row * v.ss);
}

// Elements of a 16-byte piece of a row as f32 numbers: eight bf16 words or four floats.
template <typename E>
struct Piece {
  static constexpr int kN = 16 / sizeof(E);
  float x[kN];
};
__device__ inline Piece<uint16_t> load_piece(const uint16_t* p) {
  const uint4 v = *reinterpret_cast<const uint4*>(p);
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  Piece<uint16_t> f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f.x[2 * i] = __uint_as_float(w[i] << 16);
    f.x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
  return f;
}
__device__ inline Piece<float> load_piece(const float* p) {
  const float4 v = *reinterpret_cast<const float4*>(p);
  return Piece<float>{{v.x, v.y, v.z, v.w}};
}

}  // namespace
}  // namespace citrus

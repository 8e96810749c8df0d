#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace citrus {

// Division by a number that is known at launch: n / divisor for 0 <= n < 2^31 by a multiplication.
struct FastDiv {
  int divisor;
  uint32_t mul;
  int shift;
  __device__ int quotient(int n) const {
    return static_cast<int>((__umulhi(static_cast<uint32_t>(n), mul) + static_cast<uint32_t>(n)) >> shift);
  }
};
inline FastDiv fast_div(int d) {
  FastDiv f{d, 0, 0};
  while ((int64_t{1} << f.shift) < d) ++f.shift;
  f.mul = static_cast<uint32_t>(((uint64_t{1} << 32) * ((uint64_t{1} << f.shift) - d)) / d + 1);
  return f;
}

}  // namespace citrus

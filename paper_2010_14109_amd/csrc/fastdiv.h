// Division by invariant integers on the device.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace ooc {

// x / d for 0 <= x < 2^31 and an invariant d >= 1 with one multiply-high
// (Granlund and Montgomery, division by invariant integers using
// multiplication, 1994): with l = ceil(log2 d) and m = floor(2^(31+l) / d) + 1,
// 2^(31+l) < m d <= 2^(31+l) + 2^l, hence floor(x m / 2^(31+l)) = floor(x / d)
// for every x < 2^31, and m < 2^32.  d = 1 takes m = 2^32 - 1 and adds one
// to x first: floor((x + 1)(2^32 - 1) / 2^32) = x for x + 1 <= 2^32.  Both
// cases are the same instructions, so a division never branches.
struct FastDiv {
  uint32_t d = 1, m = 0xffffffffu, s = 0, a = 1;
  static FastDiv make(int64_t dv) {
    FastDiv f;
    f.d = (uint32_t)dv;
    if (dv <= 1) return f;
    uint32_t l = 0;
    while ((1ull << l) < (uint64_t)dv) ++l;
    f.m = (uint32_t)((1ull << (31 + l)) / (uint64_t)dv + 1);
    f.s = l - 1;
    f.a = 0;
    return f;
  }
  __device__ int div(int x) const { return (int)(__umulhi((uint32_t)x + a, m) >> s); }
};

}  // namespace ooc

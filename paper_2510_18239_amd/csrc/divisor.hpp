// Division by a number that the host knows, without the dozens of instructions that a division takes on the GPU.
#pragma once

#include <cstdint>

#ifdef __HIPCC__
#define LIME_BOTH __host__ __device__
#else
#define LIME_BOTH
#endif

namespace lime {

// Of numbers below 2^31: with s = ceil(log2 d) and m = floor(2^(31 + s) / d) + 1, n / d is (n m) >> (31 + s), because m d exceeds
// 2^(31 + s) by at most d <= 2^s and n is below 2^31.
struct Divisor {
  uint32_t d = 1, m = 0x80000001u;
  int s = 0;
  LIME_BOTH Divisor() {}
  explicit Divisor(uint32_t by) : d(by) {
    while ((uint64_t{1} << s) < d) ++s;
    m = static_cast<uint32_t>((uint64_t{1} << (31 + s)) / d + 1);
  }
  LIME_BOTH int divide(int n) const {
    return static_cast<int>(static_cast<uint32_t>((static_cast<uint64_t>(static_cast<uint32_t>(n) * 2u) * m) >> 32) >> s);
  }
};

}  // namespace lime

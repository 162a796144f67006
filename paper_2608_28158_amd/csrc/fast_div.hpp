// Division of numbers below 2^31 by one that is fixed for a launch, as a
// multiplication: a division takes the GPU some 30 instructions in a chain of
// about 200 cycles, and a small call's waves begin with several.
//   s = ceil(log2 d),  m = floor(2^(31 + s) / d) + 1 <= 2^32 - 1 + 1/d,  n / d = (n m) >> (31 + s):
// n m / 2^(31 + s) exceeds n / d by at most n / 2^(31 + s) < 2^-s <= 1 / d, which
// reaches no further whole number.
#pragma once

#include <cstdint>

#if defined(__HIPCC__)
#define HARTS_HD __host__ __device__
#else
#define HARTS_HD
#endif

namespace harts {

struct FastDiv {
  uint32_t d = 1, m = 0x80000001u, s = 31;   // s: the whole shift
  FastDiv() = default;
  HARTS_HD FastDiv(uint32_t d_, uint32_t m_, uint32_t s_) : d(d_), m(m_), s(s_) {}
  explicit FastDiv(uint32_t d_) : d(d_) {
    s = 31;
    while ((uint64_t{1} << (s - 31)) < d) ++s;
    m = static_cast<uint32_t>((uint64_t{1} << s) / d + 1);
  }
  HARTS_HD inline uint32_t div(uint32_t n) const { return static_cast<uint32_t>((uint64_t{n} * m) >> s); }
  HARTS_HD inline uint32_t mod(uint32_t n) const { return n - div(n) * d; }
};

}  // namespace harts

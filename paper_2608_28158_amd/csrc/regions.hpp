// Memory that a call reads and writes, for the checks that its outputs overlap
// no other argument (host only).
#pragma once

#include <cstddef>
#include <cstdint>
#include <initializer_list>

namespace harts {

struct Region {
  const void* p;
  size_t bytes;
};

inline bool overlap(const Region& a, const Region& b) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
  return a.p && b.p && a.bytes > 0 && b.bytes > 0 && x < y + b.bytes && y < x + a.bytes;
}

inline bool overlaps_any(const Region& a, std::initializer_list<Region> others) {
  for (const Region& b : others)
    if (overlap(a, b)) return true;
  return false;
}

}  // namespace harts

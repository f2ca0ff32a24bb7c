// Host-side argument checks shared by the entry points.
#pragma once
#include <limits.h>
#include <stdint.h>

#include <initializer_list>

#include "../../include/netfuse.h"

namespace nf {

inline bool is_dtype(int dt) { return dt == NF_F32 || dt == NF_BF16; }
inline bool aligned(const void* p, size_t a) { return p == nullptr || ((uintptr_t)p % a) == 0; }

// product of non-negative ints, saturating at LLONG_MAX
inline long long prod(std::initializer_list<long long> v) {
  long long r = 1;
  for (long long x : v) {
    if (x < 0) return -1;
    if (x != 0 && r > LLONG_MAX / x) return LLONG_MAX;
    r *= x;
  }
  return r;
}
constexpr long long kMaxElems = (1LL << 62);     // element counts must stay below this
constexpr long long kMaxGrid = 0x7fffffffLL;
// HIP counts the threads of a grid in 32 bits: whether it takes so many workgroups of so many threads
inline bool grid_fits(long long blocks, int threads) { return blocks <= 0xffffffffLL / threads; }

}  // namespace nf

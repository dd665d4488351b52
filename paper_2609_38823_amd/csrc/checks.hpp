// Host-side argument checks shared by the exported entry points (after the
// header that declares moe_dtype and the status codes).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <initializer_list>

namespace decomoe {
namespace checks {

struct Range {
  uintptr_t lo, hi;  // [lo, hi)
};
inline Range rng(const void* p, size_t bytes) {
  uintptr_t a = reinterpret_cast<uintptr_t>(p);
  return Range{a, a + bytes};
}
inline bool overlap(Range a, Range b) {
  if (a.lo == a.hi || b.lo == b.hi || !a.lo || !b.lo) return false;
  return a.lo < b.hi && b.lo < a.hi;
}
// true if any output overlaps any input or another output
inline bool any_alias(std::initializer_list<Range> outs, std::initializer_list<Range> ins) {
  for (auto o = outs.begin(); o != outs.end(); ++o) {
    for (const Range& i : ins)
      if (overlap(*o, i)) return true;
    for (auto o2 = o + 1; o2 != outs.end(); ++o2)
      if (overlap(*o, *o2)) return true;
  }
  return false;
}
inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool aligned_all(std::initializer_list<const void*> ps) {
  for (const void* p : ps)
    if (p && !aligned16(p)) return false;
  return true;
}
inline int elt_size(moe_dtype dt) { return dt == MOE_BF16 ? 2 : 4; }
inline bool valid_dtype(moe_dtype dt) { return dt == MOE_F32 || dt == MOE_BF16; }
inline int hip_status(hipError_t e) { return e == hipSuccess ? MOE_OK : MOE_EHIP; }
inline size_t a256(size_t b) { return (b + 255) & ~size_t(255); }

}  // namespace checks
}  // namespace decomoe

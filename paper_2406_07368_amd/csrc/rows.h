// Checks that the C-ABI layers of the operators with strides per tensor share.
#pragma once
#include <initializer_list>

#include "../../include/linattn.h"
#include "decay.h"

namespace linattn {

constexpr int32_t kMaxTokens = 1 << 30;           // tile borders beyond the last token still fit 32 bits

inline bool finite(float x) { return x - x == 0.f; }

inline bool aligned16_all(std::initializer_list<const void*> ptrs) {
  for (const void* p : ptrs)
    if (reinterpret_cast<uintptr_t>(p) & 15u) return false;
  return true;
}

// Multiples of 8 (16-byte requests), the token axis inside a tile with 32 bits, the last row with 63.
inline bool good_input(const linattn_strides& s, int64_t B, int64_t H, int64_t L) {
  if (s.b < 0 || s.h < 0 || s.t < 0 || s.t > (int64_t)1 << 22 || ((s.b | s.h | s.t) & 7)) return false;
  return (double)s.b * (double)B + (double)s.h * (double)H + (double)s.t * (double)L < 4.0e18;
}
// ... and no two rows at the same place along one axis
inline bool good_output(const linattn_strides& s, int64_t B, int64_t H, int64_t L, int64_t d) {
  return good_input(s, B, H, L) && (L < 2 || s.t >= d) && (H < 2 || s.h >= d) && (B < 2 || s.b >= d);
}

inline Rows rows(const void* p, const linattn_strides& s) { return {p, s.b, s.h, s.t}; }

}  // namespace linattn

// Argument checks that the host dispatch of several entry points shares.
#pragma once
#include "kernels.h"

namespace linattn {
namespace checks {

inline bool misaligned(const void* p, uintptr_t to = 16) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }
inline bool overlaps(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return a && b && x < y + nb && y < x + na;
}

// Whether one of `outs` overlaps another or one of `ins`.
struct Region {
  const void* p;
  size_t bytes;
};
template <int NO, int NI>
bool any_overlap(const Region (&outs)[NO], const Region (&ins)[NI]) {
  for (int i = 0; i < NO; ++i) {
    for (const Region& in : ins)
      if (overlaps(outs[i].p, outs[i].bytes, in.p, in.bytes)) return true;
    for (int j = i + 1; j < NO; ++j)
      if (overlaps(outs[i].p, outs[i].bytes, outs[j].p, outs[j].bytes)) return true;
  }
  return false;
}

// Strides of a token tensor of H heads; bhnd: [B, H, n, d], else [B, n, H, d].
inline Rows token_rows(int H, int n, int d, bool bhnd) {
  if (bhnd) return Rows{(size_t)H * n * d, (size_t)n * d, (size_t)d};
  return Rows{(size_t)n * H * d, (size_t)d, (size_t)H * d};
}

}  // namespace checks
}  // namespace linattn

// What the entry points check of their arguments before anything is launched.
#pragma once
#include <stddef.h>
#include <stdint.h>

namespace sla2 {

inline bool misaligned16(const void* p) { return ((uintptr_t)p & 15u) != 0; }

inline bool overlaps(const void* a, size_t na, const void* b, size_t nb) {
  uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return x < y + nb && y < x + na;
}

// Two tensors of the same strides whose address ranges interleave: they are disjoint when every `period` elements (a stride that all
// larger ones are multiples of) hold each of them in its own stretch of `extent` elements, and the two stretches do not meet (nor wrap).
inline bool stretches_disjoint(const void* a, const void* b, long long esz, long long period, long long extent) {
  if (extent > period) return false;
  const long long bytes = (long long)(intptr_t)b - (long long)(intptr_t)a;
  if (bytes % esz) return false;
  const long long delta = bytes / esz, r = ((delta % period) + period) % period;
  return r >= extent && r <= period - extent;
}

}  // namespace sla2

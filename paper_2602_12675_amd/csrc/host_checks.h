// What the entry points check of their arguments before anything is launched.
#pragma once
#include <stddef.h>
#include <stdint.h>

#include "../../include/sla2.h"

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

inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// A strided tensor: `inner` neighbouring elements, `dims` times repeated.
struct View {
  const void* p;
  int esz, dims;
  long long inner, count[3], stride[3];
  size_t bytes() const {
    long long n = inner;
    for (int i = 0; i < dims; i++) n += (count[i] - 1) * stride[i];
    return (size_t)n * esz;
  }
  bool same_layout(const View& o) const {
    if (esz != o.esz || inner != o.inner || dims != o.dims) return false;
    for (int i = 0; i < dims; i++)
      if (count[i] != o.count[i] || (count[i] > 1 && stride[i] != o.stride[i])) return false;
    return true;
  }
};
inline View flat(const void* p, int esz, long long n) { return View{p, esz, 0, n, {}, {}}; }

// Slices of the rows of one buffer that hold different numbers of heads: the largest stride, that of a row, is the same, and what each
// has of a row lies in its own stretch of it.
inline bool rows_apart(const View& a, const View& b) {
  long long period[2] = {0, 0}, extent[2];
  const View* v[2] = {&a, &b};
  for (int t = 0; t < 2; t++) {
    for (int i = 0; i < v[t]->dims; i++)
      if (v[t]->count[i] > 1 && v[t]->stride[i] > period[t]) period[t] = v[t]->stride[i];
    extent[t] = v[t]->inner;
    for (int i = 0; i < v[t]->dims; i++)
      if (v[t]->count[i] > 1 && v[t]->stride[i] < period[t]) extent[t] += (v[t]->count[i] - 1) * v[t]->stride[i];
  }
  if (a.esz != b.esz || !period[0] || period[0] != period[1]) return false;
  const long long bytes = (long long)(intptr_t)b.p - (long long)(intptr_t)a.p;
  if (bytes % a.esz) return false;
  const long long r = (bytes / a.esz % period[0] + period[0]) % period[0];
  return r >= extent[0] && r + extent[1] <= period[0];
}

// Whether two tensors may share an element.  Slices of one buffer, of the same layout, interleave: they are apart if at one of the
// strides they are, what that stride repeats being the smaller ones' extent.
inline bool may_meet(const View& a, const View& b) {
  if (!a.p || !b.p || !overlaps(a.p, a.bytes(), b.p, b.bytes())) return false;
  if (!a.same_layout(b)) return !rows_apart(a, b);
  for (int k = 0; k < a.dims; k++) {
    if (a.count[k] == 1) continue;
    long long extent = a.inner;
    bool multiple = true;
    for (int i = 0; i < a.dims; i++) {
      if (i == k || a.count[i] == 1) continue;
      if (a.stride[i] < a.stride[k]) extent += (a.count[i] - 1) * a.stride[i];
      else multiple = multiple && a.stride[i] % a.stride[k] == 0;
    }
    if (multiple && stretches_disjoint(a.p, b.p, a.esz, a.stride[k], extent)) return false;
  }
  return true;
}

struct Output {
  View v;
  const void* in_place[2];                   // the inputs that it may be, where these have its layout
};
// No output on an input, unless it is that input as a whole and may be, and none on another output.  A workspace is an output.
inline bool aliased(const Output* out, int outs, const View* in, int ins) {
  for (int i = 0; i < outs; i++) {
    const Output& o = out[i];
    for (int j = 0; j < ins; j++) {
      if (!may_meet(o.v, in[j])) continue;
      const bool whole = o.v.p == in[j].p && o.v.same_layout(in[j]) && (o.v.p == o.in_place[0] || o.v.p == o.in_place[1]);
      if (!whole) return true;
    }
    for (int j = 0; j < i; j++)
      if (may_meet(o.v, out[j].v)) return true;
  }
  return false;
}

// Sum of (count - 1) stride + inner as 128 bits: whether it can be an extent in memory.
inline bool extent_ok(int dims, const long long* count, const long long* stride, long long inner) {
  __int128 n = inner;
  for (int i = 0; i < dims; i++) n += (__int128)(count[i] - 1) * stride[i];
  return n < ((__int128)1 << 60);
}

inline int check_workspace(size_t need, const void* ws, size_t bytes) {
  return !ws || ((uintptr_t)ws & 255) || bytes < need ? SLA2_EWORKSPACE : SLA2_OK;
}

}  // namespace sla2

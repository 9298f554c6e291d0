// Host checks of rows named by strides, shared by the entry points that take them.
#pragma once

#include <algorithm>

#include "rows.h"

namespace innerq {

inline bool misaligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

inline int check_rows(const void* p, const innerq_strides_t* s, int unit = 8) {
  if (!p || !s) return INNERQ_E_NULL;
  if (misaligned(p)) return INNERQ_E_ALIGN;
  for (const int64_t x : {s->batch, s->head, s->token}) {
    if (x < 0) return INNERQ_E_ARG;
    if (x % unit != 0) return INNERQ_E_ALIGN;
  }
  return INNERQ_OK;
}
// Rows that are written: none overlaps another (each dimension lies beyond the extent of those of smaller strides).
inline int check_rows_out(const void* p, const innerq_strides_t* s, long long batch, long long heads, long long tokens, int unit = 8) {
  const int st = check_rows(p, s, unit);
  if (st != INNERQ_OK) return st;
  struct Dim { int64_t stride; long long n; } dims[3] = {{s->batch, batch}, {s->head, heads}, {s->token, tokens}};
  std::sort(dims, dims + 3, [](const Dim& x, const Dim& y) { return x.stride < y.stride; });
  int64_t extent = kHeadDim;                             // elements from the first to the last of the dimensions so far
  for (const Dim& d : dims) {
    if (d.n <= 1) continue;
    if (d.stride < extent || d.stride > (INT64_MAX - extent) / (d.n - 1)) return INNERQ_E_ARG;
    extent += d.stride * (d.n - 1);
  }
  return INNERQ_OK;
}
inline RowView rows_of(const void* p, const innerq_strides_t& s) { return {static_cast<const __half*>(p), s.batch, s.head, s.token}; }

}  // namespace innerq

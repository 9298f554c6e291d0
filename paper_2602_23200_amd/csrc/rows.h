// What the calls over several new tokens of a sequence share: rows named by strides, the rotation's arguments, launchers.
#pragma once

#include "innerq_dev.h"

namespace innerq {

// Rows where a projection left them; strides in elements.
struct RowView {
  const __half* p;
  long long batch, head, token;
};

struct RotArgs {
  const float* cos;                    // null: no rotation
  const float* sin;
  const int* positions;                // [n_axes][B][t_new], or null: the token's place in its sequence
  long long axis_stride;               // B * t_new
  unsigned long long axis_low, axis_high;   // bit i: low and high bit of pair i's axis
  int last_position;                   // table_positions - 1
  int pairs, interleaved;
};

struct RotateArgs {
  RotArgs rot;
  RowView x;
  __half* y;
  long long y_batch, y_head, y_token;
  int batch, n_heads, t_new, heads_per_block;
  int n_tokens;                        // cached tokens where n_dev is null
  const int* n_dev;
  const int* t_dev;
};
hipError_t launch_rotate(const RotateArgs& a, hipStream_t stream);

// An append of up to t_new tokens a sequence.  q: the cache's tensors as an ordinary append has them (q.n_dev, q.n_old: cached
// tokens; the jobs' x_new, row_begin, row_end, ring_from and normalise are not used).
struct AppendArgs {
  QuantArgs q;
  RotArgs rot;
  RowView k, v;
  const int* t_dev;                    // new tokens of every sequence, or null: t_new
  int t_new;
  int ahead;                           // steps that the store is run ahead of the cache: 0, or 1 (ragged)
};
// counts (may be null): the caller's counters, advanced by every sequence's new tokens when all else is done.
hipError_t launch_append_rows(const AppendArgs& a, int* counts, hipStream_t stream);

}  // namespace innerq

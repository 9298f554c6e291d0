// Attention of several new tokens of a sequence to the quantised cache and, causally, to each other: arguments and launchers.
#pragma once

#include "chunk_plan.h"
#include "rows.h"

namespace innerq {

struct ChunkTensor {
  const uint8_t* codes;
  const __half* scales;
  const __half* zeros;                 // of a symmetric tensor, which has none: its scales (read, never used)
  const __half* sink;
  const __half* ring;
  RowView fresh;                       // new rows
  int slots;
};
struct ChunkArgs {
  ChunkTensor k, v;
  RowView q;
  const float* q_scale;
  void* out;
  long long out_batch, out_head, out_token;
  int out_is_fp32;
  int batch, n_q_heads, n_kv_heads, heads_per_kv, w_sink, w_recent;
  long long capacity;
  int t_new;
  int n_tokens;                        // cached, where n_dev is null
  const int* n_dev;
  const int* t_dev;
  int row_blocks, n_splits;
  float* ws_ml;                        // [B Hk][rows][n_splits][2], level in the log2 domain and sum
  float* ws_o;                         // [B Hk][rows][n_splits][d]
  PageMap pages;
};
hipError_t launch_chunk_g32(const ChunkArgs& a, int kb, int vb, const ChunkForm& form, hipStream_t stream);
hipError_t launch_chunk_g64(const ChunkArgs& a, int kb, int vb, const ChunkForm& form, hipStream_t stream);
hipError_t launch_chunk_merge(const ChunkArgs& a, hipStream_t stream);

}  // namespace innerq

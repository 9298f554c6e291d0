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
  int row_blocks, n_splits;            // the same for all sequences (without a list)
  int* table;                          // a list: first slot and splits of every sequence are left here for the merge; else null
  int list_groups;                     // work-groups of the launch
  int rows_from, rows_to;              // sequences of this launch: with that many rows (from excluded, to included)
  float* ws;                           // slots: (level in the log2 domain, sum) of every row, then 128 sums of every row
  long long slots;                     // that ws holds
  float* ws_few;                       // merge of a list: the slots of the sequences of few rows (ws: of the others)
  PageMap pages;
};
hipError_t launch_chunk_g32(const ChunkArgs& a, int kb, int vb, const ChunkForm& form, hipStream_t stream);
hipError_t launch_chunk_g64(const ChunkArgs& a, int kb, int vb, const ChunkForm& form, hipStream_t stream);
hipError_t launch_chunk_merge(const ChunkArgs& a, const ChunkForm& form, hipStream_t stream);   // form: of the launch (without a list)

}  // namespace innerq

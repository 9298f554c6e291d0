// The cache in 8 bits with a scale for each block of tokens and head: arguments and launchers of its kernels.
#pragma once

#include "block_plan.h"
#include "rows.h"

namespace innerq {

struct BlockTensor {
  uint8_t* codes;
  float* scales;
  __half* open;
};
// What all its kernels take.
struct BlockStore {
  BlockTensor k, v;
  int batch, n_kv_heads, block;
  long long capacity;
  int n_tokens;                        // cached, where n_dev is null
  const int* n_dev;
  const int* t_dev;                    // rows of every sequence, or null: t_new
  int t_new;
  PageMap pages;
};

// Number, in the code buffers, of 32-token tile `tile` of a sequence's kv head.
__device__ __forceinline__ long long block_tile(const BlockStore& s, int b, int h, int tile) {
  if (!s.pages.table) return ((long long)b * s.n_kv_heads + h) * (s.capacity / kBlockTile) + tile;
  int page = s.pages.table[(long long)b * s.pages.tiles_per_seq + (tile >> 1)];
  page = page < 0 ? 0 : page >= s.pages.pool_pages ? s.pages.pool_pages - 1 : page;
  return ((long long)page * s.n_kv_heads + h) * (kPageTokens / kBlockTile) + (tile & 1);
}
// Number of the scale of such a tile.
__device__ __forceinline__ long long block_scale(const BlockStore& s, long long tile) { return s.block == 64 ? tile >> 1 : tile; }

struct BlockAppendArgs {
  BlockStore s;
  RowView k, v;
  int units;                           // blocks of a kv head that a launch has room for
};
// counts (may be null): the caller's counters, advanced by what every sequence takes.
hipError_t launch_block_append(const BlockAppendArgs& a, int* counts, bool e4m3, hipStream_t stream);

struct BlockReadArgs {
  BlockStore s;                        // (t_new: rows)
  __half *k, *v;                       // either may be null
  long long k_batch, k_head, k_token, v_batch, v_head, v_token;
  int first;                           // where first_dev is null
  const int* first_dev;
};
hipError_t launch_block_read(const BlockReadArgs& a, bool e4m3, hipStream_t stream);

struct BlockAttnArgs {
  BlockStore s;
  RowView k, v;                        // new rows (null: cross attention)
  RowView q;
  void* out;
  long long out_batch, out_head, out_token;
  int out_is_fp32;
  int heads_per_kv;
  int row_blocks, n_splits;
  int* table;                          // a list: first slot and splits of every sequence are left here for the merge; else null
  int list_few, list_many;             // work-groups of either kind
  float* ws;                           // slots: (level in the log2 domain, sum) of every row, then 128 sums of every row
  long long slots;                     // that ws holds
  float* ws_few;                       // a ragged batch with both kinds: the slots of the sequences of few rows (ws: of the others)
  long long few_slots;
  int few_rows, few_most;              // rows of such a slot; most rows of a sequence that has them
};
hipError_t launch_block_attention(const BlockAttnArgs& a, bool e4m3, const BlockForm& form, hipStream_t stream);
hipError_t launch_block_rows(const BlockAttnArgs& a, bool e4m3, const BlockForm& form, hipStream_t stream);
hipError_t launch_block_list(const BlockAttnArgs& a, bool e4m3, hipStream_t stream);     // both kinds, with lists or without
hipError_t launch_block_merge(const BlockAttnArgs& a, const BlockForm& form, hipStream_t stream);

}  // namespace innerq

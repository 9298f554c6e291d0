// The cache in 8 bits with block scales: its arithmetic, and the launch plan of the attention over it.  Host arithmetic on sizes alone
// (no HIP); what kernels work out from counts in device memory is constexpr.
#pragma once

#include "plan.h"

namespace innerq {

constexpr int kBlockTile = 32;          // tokens that a wavefront takes at once: 4096 bytes of codes of either tensor
constexpr int kBlockTileBytes = kBlockTile * kHeadDim;
constexpr long long kBlockMostCapacity = 1LL << 24;      // tokens and their products with head_dim are 32-bit

// Tokens of n that are packed.
constexpr long long block_packed(long long n, int block) { return n - n % block; }

// ---- attention.  A row: one query head of one new token; the rows of a kv head share its keys.

constexpr int kBlockWaves = 4;          // wavefronts of a work-group, each with tiles of its own and the same rows
constexpr int kBlockSplitMost = 256;    // most ranges the keys of a row are split into

// Rows of a work-group.  Up to 64: its wavefronts have tiles of their own; more: each has a quarter of the rows.
inline int block_rows(long long rows) { return rows <= 16 ? 16 : rows <= 32 ? 32 : rows <= 64 ? 64 : rows <= 128 ? 128 : 256; }
constexpr int kBlockFewRows = 64;
// Work-groups of that form that the chip holds at once.
inline int block_round(int rows) { return rows == 64 || rows == 256 ? 256 : 512; }

struct BlockSizes {
  long long heads, rows, row_blocks;    // sequence-heads of the cache; rows of one; work-groups that they take
  int group_rows;                       // rows of a work-group
  int split_most;                       // most splits
};
inline BlockSizes block_sizes(const innerq_block_config_t& c, long long t_new) {
  BlockSizes s;
  s.heads = (long long)c.batch * c.n_kv_heads;
  s.rows = t_new * (c.n_q_heads / c.n_kv_heads);
  s.group_rows = block_rows(s.rows);
  s.row_blocks = ceil_div(s.rows, s.group_rows);
  long long most = (s.group_rows > kBlockFewRows ? 2 : 1) * block_round(s.group_rows) / (s.heads * s.row_blocks);
  most = most > kBlockSplitMost ? kBlockSplitMost : most;
  s.split_most = (int)(most < 1 ? 1 : most);
  return s;
}
// Splits of the keys (tokens: the most a row attends to).  Few rows: not shorter than two tiles a wavefront.  Many: the least rounds x (units a
// split + what a work-group costs besides).
inline int block_splits(const BlockSizes& s, long long tokens) {
  if (s.group_rows <= kBlockFewRows) {
    const long long most = ceil_div(tokens, 2LL * kBlockTile * kBlockWaves);
    return (int)(most < s.split_most ? most < 1 ? 1 : most : s.split_most);
  }
  const long long units = ceil_div(tokens, kBlockTile);
  long long best = 1, best_cost = -1;
  for (long long n = 1; n <= s.split_most && n <= units; ++n) {
    const long long rounds = ceil_div(s.heads * s.row_blocks * n, block_round(s.group_rows));
    const long long cost = rounds * (ceil_div(units, n) + 8) + (n > 1 ? 6 : 0);
    if (best_cost < 0 || cost < best_cost) { best = n; best_cost = cost; }
  }
  return (int)best;
}
// A partial result of a work-group (a slot): level, sum and 128 sums of every row.
inline size_t block_slot_bytes(int group_rows) { return (size_t)group_rows * (kHeadDim + 2) * sizeof(float); }
inline size_t block_workspace_bytes(const innerq_block_config_t& c, long long t_new) {
  const BlockSizes s = block_sizes(c, t_new);
  return 256 + (s.split_most == 1 ? 0 : (size_t)(s.heads * s.row_blocks * s.split_most) * block_slot_bytes(s.group_rows));
}

}  // namespace innerq

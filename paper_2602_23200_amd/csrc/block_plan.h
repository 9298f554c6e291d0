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

// A ragged batch of up to kBlockListMost sequences: work-groups find their work in a list made from the counts, one launch for the sequences of few
// rows and one for those of more.  kBlockListItems: work-groups that such a launch aims at, one round.
constexpr int kBlockListMost = 256;
constexpr int kBlockListItems = 512;
constexpr int kBlockListRows = 128;     // rows of a work-group of the second launch
constexpr int kBlockTableBytes = 2 * kBlockListMost * (int)sizeof(int);   // first slot and splits of every sequence, at the workspace's start
struct BlockList {
  int few_rows;                         // rows of a work-group of the first launch
  long long few, many;                  // most work-groups of either (none: 0)
};
inline BlockList block_list(const innerq_block_config_t& c, long long t_new) {
  const long long rows = t_new * (c.n_q_heads / c.n_kv_heads), heads = (long long)c.batch * c.n_kv_heads;
  const long long blocks = heads * ceil_div(rows, kBlockListRows);
  return {rows > kBlockFewRows ? kBlockFewRows : block_rows(rows), heads > kBlockListItems ? heads : kBlockListItems,
          rows <= kBlockFewRows ? 0 : blocks > kBlockListItems ? blocks : kBlockListItems};
}
// What every work-group of such a launch works out for itself (constexpr: device code, too).  A sequence's share of a launch: units, each a kv head
// and a block of `block` rows, and tiles of its keys (one, if there are none: zeros are written); none if its rows are not above `from` and up to `to`.
struct BlockShare { int units, tiles; };
constexpr BlockShare block_share(int cached, int fresh, bool causal, int heads_per_kv, int n_kv_heads, int from, int to, int block) {
  const int rows = fresh * heads_per_kv;
  if (rows <= from || rows > to) return {0, 0};
  const int tiles = (cached + (causal ? fresh : 0) + kBlockTile - 1) / kBlockTile;
  return {n_kv_heads * ((rows + block - 1) / block), tiles < 1 ? 1 : tiles};
}
// The keys of a unit are cut into ranges of `length` tiles, the same for all sequences: the first of these lengths with which the ranges are no
// more than kBlockListItems, or that of the longest sequence, which cuts none.  work: tiles of all units.
constexpr int kBlockListLeast = 8;      // (a range shorter than that is mostly set-up)
constexpr int block_first_length(float work) {
  const float even = work * (1.0f / kBlockListItems);
  return even < kBlockListLeast ? kBlockListLeast : even > 0x1p20f ? 1 << 20 : (int)even;
}
constexpr int block_next_length(int length) { return length + 1 + length / 16; }
constexpr int block_ranges(int tiles, int length) { return (tiles + length - 1) / length; }
constexpr bool block_length_fits(int length, int longest, int ranges) { return length >= longest || ranges <= kBlockListItems; }
// Range number `at` of a sequence: row blocks of the same range, which read the same keys, are neighbours.
struct BlockPlace { int h, row_block, split; };
constexpr BlockPlace block_place(int at, int units, int n_kv_heads, int splits) {
  const int blocks = units / n_kv_heads, h = at / (blocks * splits), rest = at - h * blocks * splits;
  return {h, rest % blocks, rest / blocks};
}

inline size_t block_workspace_bytes(const innerq_block_config_t& c, long long t_new) {
  const BlockSizes s = block_sizes(c, t_new);
  size_t bytes = s.split_most == 1 ? 0 : (size_t)(s.heads * s.row_blocks * s.split_most) * block_slot_bytes(s.group_rows);
  if (c.batch <= kBlockListMost) {
    // (work-groups beyond the items that were aimed at have no partial results: their sequences are not split)
    const BlockList l = block_list(c, t_new);
    const size_t list = (size_t)kBlockListItems * (block_slot_bytes(l.few_rows) + (l.many ? block_slot_bytes(kBlockListRows) : 0));
    bytes = list > bytes ? list : bytes;
  }
  return kBlockTableBytes + bytes;
}

}  // namespace innerq

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

constexpr int kBlockSplitMost = 256;    // most ranges the keys of a row are split into

// A work-group: its rows, and wavefronts.  Up to 64 rows: the wavefronts have tiles of their own; more: each has a part of the rows.
struct BlockForm { int rows, waves; };
constexpr int kBlockFewRows = 64;
// 16 rows: eight wavefronts leave fewer partial results where sequence-heads are few, four share the chip better where they are many (us, four and
// eight: one token of 8 heads x 32k 25.7, 20.0; 32 x 8k 19.7, 17.9; 256 x 8k 84.8, 81.3; 512 x 1437 33.3, 35.7; 512 x 90 to 1437 17.5, 21.4).
constexpr BlockForm block_form(long long rows, long long heads) {
  if (rows <= 16) return {16, heads > 256 ? 4 : 8};
  return rows <= 32 ? BlockForm{32, 4} : rows <= 64 ? BlockForm{64, 4} : rows <= 128 ? BlockForm{128, 4} : BlockForm{256, 8};
}
// Work-groups of that form that the chip holds at once.
constexpr int block_round(const BlockForm& f) { return f.rows == 16 ? (f.waves == 4 ? 768 : 256) : f.rows == 32 || f.rows == 128 ? 512 : 256; }

struct BlockSizes {
  long long heads, rows, row_blocks;    // sequence-heads of the cache; rows of one; work-groups that they take
  BlockForm form;
  int split_most;                       // most splits
};
inline BlockSizes block_sizes(const innerq_block_config_t& c, long long t_new) {
  BlockSizes s;
  s.heads = (long long)c.batch * c.n_kv_heads;
  s.rows = t_new * (c.n_q_heads / c.n_kv_heads);
  s.form = block_form(s.rows, s.heads);
  s.row_blocks = ceil_div(s.rows, s.form.rows);
  long long most = (s.form.rows > kBlockFewRows ? 2 : 1) * block_round(s.form) / (s.heads * s.row_blocks);
  most = most > kBlockSplitMost ? kBlockSplitMost : most;
  s.split_most = (int)(most < 1 ? 1 : most);
  return s;
}
// Splits of the keys (tokens: the most a row attends to).  Few rows: the least tiles a wavefront, a second launch for the splits counted as four of
// them.  Many: the least rounds x (units a split + what a work-group costs besides).
inline int block_splits(const BlockSizes& s, long long tokens) {
  const long long units = ceil_div(tokens, kBlockTile);
  long long best = 1, best_cost = -1;
  for (long long n = 1; n <= s.split_most && n <= units; ++n) {
    const long long rounds = ceil_div(s.heads * s.row_blocks * n, block_round(s.form));
    const long long cost = s.form.rows <= kBlockFewRows ? ceil_div(units, n * s.form.waves) + (n > 1 ? 4 : 0)
                                                         : rounds * (ceil_div(units, n) + 8) + (n > 1 ? 6 : 0);
    if (best_cost < 0 || cost < best_cost) { best = n; best_cost = cost; }
  }
  return (int)best;
}
// A partial result of a work-group (a slot): level, sum and 128 sums of every row.
inline size_t block_slot_bytes(int group_rows) { return (size_t)group_rows * (kHeadDim + 2) * sizeof(float); }

// A ragged batch of up to kBlockListMost sequences: work-groups find their work in two lists made from the counts, of the sequences of few rows and of
// those of more, each aimed at one round of work-groups.  With both they are one launch, the work-groups of many rows first: those of few rows find room
// beside them and wait for memory while they compute (two launches and this one: 16 sequences of 1 to 256 new tokens over 1 to 16k 182 us, 167; 8 of 1 to
// 40 over 1 to 4000 41.4, 32.2; 64 of 1 to 512 566, 551).  Sequences of few rows alone that fill half a round as they are have no list: it costs 4 us
// in front of the first load, and a launch behind.  The second list's work-groups have 128 rows, not 256, and the first one's up to 32, not 64 (the
// first of these cases, in two launches: 199 and 215 us; 187 and 199).
constexpr int kBlockListMost = 256;
constexpr int kBlockListFew = 32;       // most rows of a sequence of the first list
constexpr BlockForm kBlockListMany = {128, 4};           // work-groups of the second list
constexpr int kBlockTableBytes = 2 * kBlockListMost * (int)sizeof(int);   // first slot and splits of every sequence, at the workspace's start
struct BlockList {
  bool use;
  BlockForm form;                       // of the first list
  long long few, many;                  // most work-groups of either (none: 0), a multiple of eight
};
constexpr BlockForm block_list_form(long long rows) { return rows <= 16 ? BlockForm{16, 4} : BlockForm{32, 4}; }
inline BlockList block_list(const innerq_block_config_t& c, long long t_new) {
  const long long rows = t_new * (c.n_q_heads / c.n_kv_heads), heads = (long long)c.batch * c.n_kv_heads;
  const long long blocks = heads * ceil_div(rows, kBlockListMany.rows);
  BlockList l;
  l.form = block_list_form(rows);
  l.few = (heads > block_round(l.form) ? heads : block_round(l.form)) + 7 & ~7LL;
  l.many = rows <= kBlockListFew ? 0 : (blocks > block_round(kBlockListMany) ? blocks : block_round(kBlockListMany)) + 7 & ~7LL;
  l.use = c.batch <= kBlockListMost && (l.many || 2 * heads <= block_round(l.form));
  return l;
}
// What every work-group works out for itself (constexpr: device code, too).  A sequence's share of a list: units, each a kv head
// and a block of `block` rows, and tiles of its keys (one, if there are none: zeros are written); none if its rows are not above `from` and up to `to`.
struct BlockShare { int units, tiles; };
constexpr BlockShare block_share(int cached, int fresh, bool causal, int heads_per_kv, int n_kv_heads, int from, int to, int block) {
  const int rows = fresh * heads_per_kv;
  if (rows <= from || rows > to) return {0, 0};
  const int tiles = (cached + (causal ? fresh : 0) + kBlockTile - 1) / kBlockTile;
  return {n_kv_heads * ((rows + block - 1) / block), tiles < 1 ? 1 : tiles};
}
// The keys of a unit are cut into ranges of `length` tiles, the same for all sequences: the first of these lengths with which the ranges are no
// more than `items`, or that of the longest sequence, which cuts none.  work: tiles of all units; ranges: with `length`.  (Ranges are work / length
// and a part of one a unit; the next length is what would fit if those parts stayed the same, or a sixteenth more.)
constexpr int kBlockListLeast = 8;      // (a range shorter than that is mostly set-up)
constexpr int block_first_length(float work, int items) {
  const float even = work / (float)items;
  return even < kBlockListLeast ? kBlockListLeast : even > 0x1p20f ? 1 << 20 : (int)even;
}
constexpr int block_next_length(int length, int ranges, int items) {
  const float fits = (float)length * (float)ranges / (float)items;
  const int least = length + 1 + length / 16;
  return fits < (float)least || !(fits < 0x1p20f) ? least : (int)fits;
}
constexpr int block_ranges(int tiles, int length) { return (tiles + length - 1) / length; }
constexpr bool block_length_fits(int length, int longest, int ranges, int items) { return length >= longest || ranges <= items; }
// Range number `at` of a sequence: row blocks of the same range, which read the same keys, are neighbours.
struct BlockPlace { int h, row_block, split; };
constexpr BlockPlace block_place(int at, int units, int n_kv_heads, int splits) {
  const int blocks = units / n_kv_heads, h = at / (blocks * splits), rest = at - h * blocks * splits;
  return {h, rest % blocks, rest / blocks};
}

inline size_t block_workspace_bytes(const innerq_block_config_t& c, long long t_new) {
  const BlockSizes s = block_sizes(c, t_new);
  size_t bytes = s.split_most == 1 ? 0 : (size_t)(s.heads * s.row_blocks * s.split_most) * block_slot_bytes(s.form.rows);
  const BlockList l = block_list(c, t_new);
  if (l.use) {
    // (work-groups beyond the round that was aimed at have no partial results: their sequences are not split)
    const size_t list = block_round(l.form) * block_slot_bytes(l.form.rows) + (l.many ? block_round(kBlockListMany) * block_slot_bytes(kBlockListMany.rows) : 0);
    bytes = list > bytes ? list : bytes;
  }
  return kBlockTableBytes + bytes;
}

}  // namespace innerq

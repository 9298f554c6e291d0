// The launch plan of an attention call over several new tokens: which work-groups, how the keys are split, how much workspace.
// Host arithmetic on sizes alone (no HIP).
#pragma once

#include "plan.h"

namespace innerq {

constexpr int kChunkWaveRows = 32;      // query rows of a wavefront (a row: one query head of one new token)
constexpr int kChunkSplitMost = 256;    // most ranges the keys of a row are split into
constexpr int kChunkListMost = 256;     // most sequences of a batch whose work is shared out by their lengths
// Work-groups that such a launch aims at: one round.  (us with 512, 1024 and 1536, 32 / 8 heads, 4 bits, counts spread over a factor of 16 and
// more: 32 sequences to 8k tokens, to 64 new 111, 135, 146; 16 to 16k, to 8 new 53, 63, 72; 4 to 16k, to 512 new 122, 141, 157; 16 to 16k, to 256
// new 244, 236, 258: more ranges share the work better and leave more partial results.)
constexpr int kChunkListItems = 512;
constexpr int kChunkTableBytes = 2 * kChunkListMost * (int)sizeof(int);   // first slot and splits of every sequence, at the workspace's start

struct ChunkForm {
  int row_waves;                        // wavefronts of a work-group that share a tile of keys, each with its own 32 rows
  int token_waves;                      // wavefronts of a work-group with tiles of their own (and the same rows)
  int tile;                             // tokens of a tile
  int round;                            // work-groups that the chip holds at once
  int rows() const { return row_waves * kChunkWaveRows; }
};
// Few rows: a wavefront has all of them, and four of a work-group share the keys.  More: four or eight wavefronts share a tile, brought to
// fp16 once for 128 or 256 rows.  Eight are the faster where most keys are packed (us, four and eight, 32 / 8 heads, 4 bits: 2048 new tokens
// over 32k 1396, 1226; over 8k 446, 405; 512 over 16k 208, 188; 256 over 16k 120, 112), four among new tokens, where a work-group's rows
// end at different ones and two work-groups a compute unit fill each other's gaps (2048 over none 72, 97; over 2048 165, 177; 4096 of 32
// heads over none 200, 215; over 4096 586, 562).
constexpr ChunkForm kFewRows = {1, 4, 32, 512}, kSomeRows = {4, 1, 64, 512}, kManyRows = {8, 1, 64, 256};
inline ChunkForm chunk_form(long long rows, long long t_new, long long cached) {
  return rows <= kChunkWaveRows ? kFewRows : rows <= 128 || cached < 2 * t_new ? kSomeRows : kManyRows;
}

struct ChunkSizes {
  ChunkForm form;
  long long heads, rows, row_blocks;    // sequence-heads of the cache; rows of one; work-groups that they take
  int split_most;                       // most splits
};
inline ChunkSizes chunk_sizes(const innerq_config_t& c, long long t_new, long long cached) {
  ChunkSizes s;
  s.heads = (long long)c.batch * c.n_kv_heads;
  s.rows = t_new * (c.n_q_heads / c.n_kv_heads);
  s.form = chunk_form(s.rows, t_new, cached);
  s.row_blocks = ceil_div(s.rows, s.form.rows());
  // up to two rounds of work-groups
  long long most = 2 * s.form.round / (s.heads * s.row_blocks);
  const long long tiles = ceil_div((long long)c.capacity_tokens, s.form.tile) + 2;
  most = most > kChunkSplitMost ? kChunkSplitMost : most;
  most = most > tiles ? tiles : most;
  s.split_most = (int)(most < 1 ? 1 : most);
  return s;
}

// Splits of the keys (tokens: the most a row attends to): the least rounds x (tiles a split + what a work-group costs besides).
inline int chunk_splits(const ChunkSizes& s, long long tokens) {
  const long long tiles = ceil_div(tokens, (long long)s.form.tile * s.form.token_waves);
  long long best = 1, best_cost = -1;
  for (long long n = 1; n <= s.split_most && n <= tiles; ++n) {
    const long long rounds = ceil_div(s.heads * s.row_blocks * n, s.form.round);
    const long long cost = rounds * (ceil_div(tiles, n) + 3) + (n > 1 ? 2 : 0);
    if (best_cost < 0 || cost < best_cost) { best = n; best_cost = cost; }
  }
  return (int)best;
}

// A partial result of a work-group (a slot): level, sum and 128 sums of every row.
inline size_t chunk_slot_bytes(const ChunkForm& f) { return (size_t)f.rows() * (kHeadDim + 2) * sizeof(float); }

// A ragged batch of up to kChunkListMost sequences: work-groups find their work in a list made from the counts, one launch for the sequences of few
// rows and one for those of more.  Most work-groups of either launch (none: 0).  Such a list has four wavefronts a tile wherever the keys are, and
// its work-groups go to any XCD: one sequence through the list and without it, us, 2048 new tokens over 32k 1420, 1226 (8 kv heads), first prompt
// of 4096 314, 205 (32).
struct ChunkList { long long few, some; };
inline ChunkList chunk_list(const innerq_config_t& c, long long t_new) {
  const long long rows = t_new * (c.n_q_heads / c.n_kv_heads), heads = (long long)c.batch * c.n_kv_heads;
  const long long blocks = heads * ceil_div(rows, kSomeRows.rows());
  return {heads > kChunkListItems ? heads : kChunkListItems, rows <= kChunkWaveRows ? 0 : blocks > kChunkListItems ? blocks : kChunkListItems};
}

// What every work-group of such a launch works out for itself (constexpr: device code, too).  A sequence's share of a launch: units, each a kv head
// and a block of `block` rows, and tiles of its keys; none if its rows are not above `from` and up to `to`.
struct ChunkShare { int units, tiles; };
constexpr ChunkShare chunk_share(int cached, int fresh, int heads_per_kv, int n_kv_heads, int from, int to, int block, int tile) {
  const int rows = fresh * heads_per_kv;
  if (rows <= from || rows > to) return {0, 0};
  return {n_kv_heads * ((rows + block - 1) / block), (cached + fresh + tile - 1) / tile};
}
// The keys of a unit are cut into ranges of `length` tiles, the same for all sequences: the first of these lengths with which the ranges are no
// more than kChunkListItems, or that of the longest sequence, which cuts none.  work: tiles of all units.
constexpr int kChunkListLeast = 4;       // (a range shorter than that is mostly set-up)
constexpr int chunk_first_length(float work) {
  // (a call's tokens are at most 2^25, so no sequence has more than 2^19 tiles; beyond, sums with a length would pass 31 bits)
  const float even = work * (1.0f / kChunkListItems);
  return even < kChunkListLeast ? kChunkListLeast : even > 0x1p20f ? 1 << 20 : (int)even;
}
constexpr int chunk_next_length(int length) { return length + 1 + length / 8; }
constexpr int chunk_ranges(int tiles, int length) { return (tiles + length - 1) / length; }
constexpr bool chunk_length_fits(int length, int longest, int ranges) { return length >= longest || ranges <= kChunkListItems; }
// Range number `at` of a sequence.
struct ChunkPlace { int h, row_block, split; };
constexpr ChunkPlace chunk_place(int at, int units, int n_kv_heads, int splits) {
  const int unit = at / splits, blocks = units / n_kv_heads, h = unit / blocks;
  return {h, unit - h * blocks, at - unit * splits};
}

inline size_t chunk_workspace_bytes(const innerq_config_t& c, long long t_new) {
  size_t bytes = 0;
  const long long either[2] = {0, 2 * t_new};            // (either form of that many rows)
  for (const long long cached : either) {
    const ChunkSizes s = chunk_sizes(c, t_new, cached);
    const size_t need = s.split_most == 1 ? 0 : (size_t)(s.heads * s.row_blocks * s.split_most) * chunk_slot_bytes(s.form);
    bytes = need > bytes ? need : bytes;
  }
  if (c.batch <= kChunkListMost) {
    // (work-groups beyond the items that were aimed at have no partial results: their sequences are not split)
    const ChunkList l = chunk_list(c, t_new);
    const size_t list = (size_t)kChunkListItems * (chunk_slot_bytes(kFewRows) + (l.some ? chunk_slot_bytes(kSomeRows) : 0));
    bytes = list > bytes ? list : bytes;
  }
  return kChunkTableBytes + bytes;
}

}  // namespace innerq

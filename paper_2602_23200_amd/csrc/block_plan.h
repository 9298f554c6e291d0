// The cache in 8 bits with block scales: its arithmetic, and the launch plan of the attention over it.  Host arithmetic on sizes alone
// (no HIP); what kernels work out from counts in device memory is constexpr.
#pragma once

#include <cmath>
#include <initializer_list>

#include "plan.h"

namespace innerq {

constexpr int kBlockTile = 32;          // tokens that a wavefront takes at once: 4096 bytes of codes of either tensor
constexpr int kBlockTileBytes = kBlockTile * kHeadDim;
constexpr long long kBlockMostCapacity = 1LL << 24;      // tokens and their products with head_dim are 32-bit

// Tokens of n that are packed.
constexpr long long block_packed(long long n, int block) { return n - n % block; }

// Eight-bit integers as fp16 times 2^x, with one rounding.  A byte of two's complement with its sign bit flipped, code + 128, is put under the exponent of 1024
// (the other byte is 0x64): the number 1024 + 128 + code, which times 2^x, and 1152 2^x taken away, is one fused operation.  Below 2^-24 the factor is no
// fp16 number any more; there the byte stands alone, as (code + 128) 2^-24, with a factor of 2^(x + 24) and 128 2^x taken away.  Below 2^-31 every
// product is less than half of the smallest step: zero.
constexpr uint32_t half_power(int x) { return x >= -14 ? (uint32_t)(x + 15) << 10 : 1u << (x + 24); }        // bits of 2^x, -24 <= x <= 15
constexpr uint32_t int_codes(int x) {                    // x <= 5; the factor in the lower half, what is taken away (as a negative number) in the upper one
  return x >= -24 ? half_power(x) | (0x8080u | (uint32_t)(x + 25) << 10) << 16 : x >= -31 ? half_power(x + 24) | (0x8000u | half_power(x + 7)) << 16 : 0u;
}
// (1152 is 1.125 x 1024: its bit stands for the case, since a power of two below 2^-17 has no bit there)
constexpr uint32_t int_codes_top(uint32_t both) { return both >> 23 & 1u ? 0x64646464u : 0u; }

// ---- attention.  A row: one query head of one new token; the rows of a kv head share its keys.
constexpr int kBlockSplitMost = 256;    // most ranges the keys of a row are split into

// A work-group: its rows, and wavefronts.  Up to 64 rows: the wavefronts have tiles of their own; more: each has a part of the rows.
struct BlockForm { int rows, waves; };
constexpr int kBlockFewRows = 64;
// Work-groups of that form that the chip holds at once.
constexpr int block_round(const BlockForm& f) { return 256 * (f.rows == 16 ? 3 : f.rows == 32 || f.rows == 128 ? 2 : 1); }

// What a form costs, us: before the first tile of the first work-groups and of later ones; for every tile that a wavefront (many rows: the work-group) takes
// one after the other, with a CU of its own and in more than 256 work-groups; where the keys are split, for the second launch and for so many rows of
// partial results.  The constants are fitted to 16700 timings of calls with 4 to 2048 rows of each of 1 to 1024 sequence-heads over 0 to 32k tokens, every
// form and number of ranges; of these the one that is chosen takes 0.9 % longer than the fastest one in the mean, 27 % at worst.  (By the number of rows
// alone, with as many ranges as fill the chip, calls of 17 rows and more took 25 % longer in the mean, three times as long at worst: 300 rows of 8 heads
// over 300 tokens 26 us, now 12; 128 over 1682 29, now 13.)
struct BlockKind { BlockForm form; float setup, again, tile, crowded, join, partial; };
constexpr BlockKind kBlockKinds[] = {{{16, 4}, 5.0f, 3.0f, 0.62f, 1.4f, 3.0f, 4200.f},
                                     {{32, 4}, 6.4f, 5.0f, 0.86f, 1.8f, 3.0f, 4200.f},
                                     {{64, 4}, 8.3f, 6.5f, 1.2f, 1.2f, 3.0f, 6300.f},
                                     {{128, 4}, 9.2f, 3.0f, 0.69f, 1.0f, 3.5f, 8400.f},
                                     {{256, 8}, 9.3f, 7.0f, 0.89f, 0.89f, 4.4f, 8400.f}};
constexpr BlockKind kBlockFew = kBlockKinds[1], kBlockMany = kBlockKinds[3];     // of a list
// Bytes of the cache a us.  (Up to 224 work-groups no CU has two while another has none.  8 sequences of 8 heads over 32k tokens, one token: in 3 ranges 84 us,
// 4 93, 6 90, 8 93, 12 91; 5 tokens: 93, 96, 97, 98.)
constexpr float block_rate(float groups) { return groups <= 224.f ? 6.5e6f : 6.0e6f; }
// Fewest rows of a form.
constexpr int block_least_rows(const BlockForm& f) { return f.rows == 16 ? 1 : f.rows / 2 + 1; }
// Forms that come into question (of 16 rows a work-group for 17 and more reads the keys too often, of 64 for 129; wider ones would be empty for the most part).
constexpr bool block_suits(const BlockForm& f, long long rows) {
  return rows >= block_least_rows(f) && (f.rows == 16 ? rows <= 16 : f.rows != 64 || rows <= 128);
}
// units: tiles of the longest row block; average: of one in the mean.
inline float block_cost(const BlockKind& k, long long heads, long long row_blocks, float units, float average, int n) {
  const float groups = (float)(heads * row_blocks) * (float)n, ways = (float)(k.form.rows <= kBlockFewRows ? n * k.form.waves : n);
  const float share = units / ways, tile = groups <= 256.f ? k.tile : k.crowded, rounds = groups / (float)block_round(k.form);
  float us = k.setup + 0.5f * (std::ceil(share) + (share < 1.f ? 1.f : share)) * tile;
  if (rounds > 1.f) {
    const float mean = average / ways, r = rounds <= 3.f ? std::ceil(rounds) : rounds + 0.5f;
    const float all = k.setup + (r - 1.f) * k.again + r * (mean < 0.5f ? 0.5f : mean) * tile;
    us = all > us ? all : us;
  }
  const float bytes = (float)heads * units * (2 * kBlockTileBytes) / block_rate(groups);
  us = std::sqrt(std::sqrt(us * us * us * us + bytes * bytes * bytes * bytes));      // (the larger of the two, and more where they are alike)
  return us + (n > 1 ? k.join + 0.85f * (float)((n + 7) / 8) + groups * (float)k.form.rows / k.partial : 0.f);
}
// Most partial results: for one round of work-groups (many rows: two).
constexpr int block_most_slots(const BlockForm& f) { return (f.rows > kBlockFewRows ? 2 : 1) * block_round(f); }
inline int block_split_most(const BlockForm& f, long long heads, long long row_blocks) {
  const long long most = block_most_slots(f) / (heads * row_blocks);
  return (int)(most < 1 ? 1 : most > kBlockSplitMost ? kBlockSplitMost : most);
}
struct BlockPlan { BlockForm form; long long row_blocks; int n_splits; float us; };
inline BlockPlan block_plan_of(const BlockKind& k, long long heads, long long rows, float units, float average) {
  BlockPlan best = {k.form, ceil_div(rows, k.form.rows), 1, 0.f};
  if (best.row_blocks == 1) average = units;
  const int most = block_split_most(k.form, heads, best.row_blocks);
  best.us = block_cost(k, heads, best.row_blocks, units, average, 1);
  // (steps of an eighth and less)
  for (int n = 2; n <= most && (float)n <= units; n += n < 8 ? 1 : n < 16 ? 2 : n < 32 ? 4 : n < 64 ? 8 : n < 128 ? 16 : 32) {
    const float us = block_cost(k, heads, best.row_blocks, units, average, n);
    if (us < best.us) { best.us = us; best.n_splits = n; }
  }
  return best;
}
// tokens: the most that a row attends to; of them, for the row block in the mean, `fewer` not.
inline BlockPlan block_plan(const innerq_block_config_t& c, long long t_new, long long tokens, float fewer) {
  const long long heads = (long long)c.batch * c.n_kv_heads, rows = t_new * (c.n_q_heads / c.n_kv_heads);
  const float units = (float)ceil_div(tokens, kBlockTile), average = units - fewer / kBlockTile;
  BlockPlan best = {};
  for (const BlockKind& k : kBlockKinds) {
    if (!block_suits(k.form, rows)) continue;
    const BlockPlan x = block_plan_of(k, heads, rows, units, average);
    if (best.n_splits == 0 || x.us < best.us) best = x;
  }
  return best;
}

// A partial result of a work-group (a slot): level, sum and 128 sums of every row.
inline size_t block_slot_bytes(int group_rows) { return (size_t)group_rows * (kHeadDim + 2) * sizeof(float); }

// A ragged batch of up to kBlockListMost sequences: work-groups find their work in two lists made from the counts, of the sequences of few rows and of
// those of more, each aimed at a number of work-groups.  With both they are one launch, the work-groups of many rows first: those of few rows find room
// beside them and wait for memory while they compute (two launches and this one: 16 sequences of 2 to 256 new tokens over 1000 to 16000 182 us,
// 167; 8 of 1 to 40 over 250 to 4000 41.4, 32.2).  Sequences of few rows alone that fill half a round as they are have no list: it costs 4 us
// in front of the first load, and a launch behind.  (Without it one token of 64 sequences of 8 heads over 500 to 8000 tokens takes 75 us, 361 MB, of 64 over 2000 to
// 32000 287, 1436 MB, of 32 of 16 heads over 500 to 8000 76, 365 MB: 4.8 to 5.0 TB/s, a copy's rate; with it 48 of 8 heads over 500 to 8000 59, 272 MB: 4.6.)  The second list's work-groups have 128 rows, not 256, and the first one's up to 32, not 64 (the
// first of these cases, in two launches: 199 and 215 us; 187 and 199).
constexpr int kBlockListMost = 256;
// Ranges that a list aims at.  (As many as the chip holds, 768, 512 and 512: 8 sequences of 2k to 32k tokens, one new one 46.8 us, with these 43.8; of 500 to
// 8000 22.7 and 21.2, 1 to 5 new ones 24.0 and 21.4; cross attention of 16 x 16 heads over 89 to 1437 17.7 and 18.7.)
constexpr int block_list_items(const BlockForm& f) { return f.rows == 32 ? 256 : 512; }
constexpr int kBlockTableBytes = 2 * kBlockListMost * (int)sizeof(int);   // first slot and splits of every sequence, at the workspace's start
struct BlockList {
  bool use;
  BlockForm form;                       // of the first list
  int few_most;                         // most rows of a sequence of the first list
  long long few, many;                  // most work-groups of either (none: 0), a multiple of eight
};
inline BlockList block_list_of(const innerq_block_config_t& c, long long t_new, bool all_few) {
  const long long rows = t_new * (c.n_q_heads / c.n_kv_heads), heads = (long long)c.batch * c.n_kv_heads;
  BlockList l;
  l.form = rows <= 16 ? kBlockKinds[0].form : kBlockFew.form;
  l.few_most = (int)(all_few || rows <= l.form.rows ? rows : l.form.rows);
  const long long few = heads * ceil_div(l.few_most, l.form.rows), many = heads * ceil_div(rows, kBlockMany.form.rows);
  l.few = (few > block_list_items(l.form) ? few : block_list_items(l.form)) + 7 & ~7LL;
  l.many = rows <= l.few_most ? 0 : (many > block_list_items(kBlockMany.form) ? many : block_list_items(kBlockMany.form)) + 7 & ~7LL;
  l.use = c.batch <= kBlockListMost && (rows > l.form.rows || 2 * few <= block_round(l.form));
  return l;
}
// Every sequence in the first list where a batch of the longest ones would be faster so.
inline BlockList block_list(const innerq_block_config_t& c, long long t_new, long long tokens) {
  const long long rows = t_new * (c.n_q_heads / c.n_kv_heads), heads = (long long)c.batch * c.n_kv_heads;
  const float units = (float)ceil_div(tokens, kBlockTile);
  const bool all_few = rows <= kBlockFew.form.rows || block_plan_of(kBlockFew, heads, rows, units, units).us <= block_plan_of(kBlockMany, heads, rows, units, units).us;
  return block_list_of(c, t_new, all_few);
}
// Larger batches have no list.  Where a sequence may have more rows than few, all have the work-groups that the longest would have, as many ranges each, and every
// work-group takes the form of its own sequence, so that what weights are rounded to does not depend on other sequences.
inline bool block_both_kinds(const innerq_block_config_t& c, long long t_new) {
  return c.batch > kBlockListMost && t_new * (c.n_q_heads / c.n_kv_heads) > kBlockFew.form.rows;
}
inline BlockPlan block_plan_both(const innerq_block_config_t& c, long long t_new, long long tokens) {
  const float units = (float)ceil_div(tokens, kBlockTile);
  return block_plan_of(kBlockMany, (long long)c.batch * c.n_kv_heads, t_new * (c.n_q_heads / c.n_kv_heads), units, units);
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
// Which range a work-group takes.  Work-groups go to the eight dies in turn.  Where heads are a multiple of eight a die has an eighth of the heads, of every
// sequence: a head's keys are read by one die, and sequences of any lengths are shared out evenly.  Otherwise a die has an eighth of the line.  (An eighth
// of the line for each die, and this: 8 prompts of 15 to 2000 tokens 152 us, 97; 64 sequences of 4 to 512 new tokens over 250 to 4000 555, 313; the 16
// above 157, 153.)  The last rows, which have the most keys, go first.
constexpr bool block_by_head(int n_kv_heads) { return n_kv_heads % 8 == 0; }
// Its place in the line (by head: in its die's line, an eighth of every sequence's ranges; none: -1).
constexpr int block_turn(int group, int ranges, bool by_head) {
  const int per = (ranges + 7) / 8, turn = group / 8, place = by_head ? turn : group % 8 * per + turn;
  return turn < per && (by_head || place < ranges) ? place : -1;
}
// The number of the range within its sequence, from its place there.
constexpr int block_range(int place, int group, int units, int n_kv_heads, int splits, bool by_head) {
  const int blocks = units / n_kv_heads, each = blocks * splits, h = by_head ? place / each * 8 + group % 8 : place / each, rest = place % each;
  return h * each + rest / blocks * blocks + blocks - 1 - rest % blocks;
}
// Range number `at` of a sequence: row blocks of the same range, which read the same keys, are neighbours.
struct BlockPlace { int h, row_block, split; };
constexpr BlockPlace block_place(int at, int units, int n_kv_heads, int splits) {
  const int blocks = units / n_kv_heads, h = at / (blocks * splits), rest = at - h * blocks * splits;
  return {h, rest % blocks, rest / blocks};
}

// Whatever the number of tokens, and enough for fewer rows, too.
inline size_t block_workspace_bytes(const innerq_block_config_t& c, long long t_new) {
  const long long heads = (long long)c.batch * c.n_kv_heads, rows = t_new * (c.n_q_heads / c.n_kv_heads);
  size_t bytes = 0;
  for (const BlockKind& k : kBlockKinds) {
    // (fewer row blocks may be split where these are not)
    const bool both = k.form.rows == kBlockMany.form.rows && block_both_kinds(c, t_new);
    if ((rows < block_least_rows(k.form) && !both) || block_split_most(k.form, heads, 1) == 1) continue;
    const size_t slots = block_most_slots(k.form) * block_slot_bytes(k.form.rows);
    bytes = slots > bytes ? slots : bytes;
  }
  for (const bool all_few : {false, true}) {
    const BlockList l = block_list_of(c, t_new, all_few);
    if (!l.use) continue;
    // (work-groups beyond the number that was aimed at have no partial results: their sequences are not split)
    const size_t list = block_list_items(l.form) * block_slot_bytes(l.form.rows) + (l.many ? block_list_items(kBlockMany.form) * block_slot_bytes(kBlockMany.form.rows) : 0);
    bytes = list > bytes ? list : bytes;
  }
  return kBlockTableBytes + bytes;
}

}  // namespace innerq

// The launch plan of an attention call over several new tokens: which work-groups, how the keys are split, how much workspace.
// Host arithmetic on sizes alone (no HIP).
#pragma once

#include "plan.h"

namespace innerq {

constexpr int kChunkWaveRows = 32;      // query rows of a wavefront (a row: one query head of one new token)
constexpr int kChunkSplitMost = 256;    // most ranges the keys of a row are split into
constexpr int kChunkGroups = 512;       // work-groups that the chip holds at once (two a compute unit): what splitting aims at

struct ChunkForm {
  int row_waves;                        // wavefronts of a work-group that share a tile of keys, each with its own 32 rows
  int token_waves;                      // wavefronts of a work-group with tiles of their own (and the same rows)
  int tile;                             // tokens of a tile
};
// Few rows: a wavefront has all of them, and four of a work-group share the keys; else four wavefronts of 32 rows share a tile.
inline ChunkForm chunk_form(long long rows) { return rows <= kChunkWaveRows ? ChunkForm{1, 4, 32} : rows <= 128 ? ChunkForm{4, 1, 64} : ChunkForm{8, 1, 64}; }

struct ChunkSizes {
  ChunkForm form;
  long long heads, rows, row_blocks;    // sequence-heads of the cache; rows of one; work-groups that they take
  int split_most;                       // most splits of the workspace
  size_t bytes;                         // of the workspace: (m, l) and 128 sums a row and split
};
inline ChunkSizes chunk_sizes(const innerq_config_t& c, long long t_new) {
  ChunkSizes s;
  s.heads = (long long)c.batch * c.n_kv_heads;
  s.rows = t_new * (c.n_q_heads / c.n_kv_heads);
  s.form = chunk_form(s.rows);
  s.row_blocks = ceil_div(s.rows, (long long)s.form.row_waves * kChunkWaveRows);
  // up to two rounds of work-groups
  long long most = 2 * kChunkGroups / (s.heads * s.row_blocks);
  const long long tiles = ceil_div((long long)c.capacity_tokens, s.form.tile) + 2;
  most = most > kChunkSplitMost ? kChunkSplitMost : most;
  most = most > tiles ? tiles : most;
  s.split_most = (int)(most < 1 ? 1 : most);
  s.bytes = s.split_most == 1 ? 64 : (size_t)s.heads * s.rows * s.split_most * (kHeadDim + 2) * sizeof(float) + 64;
  return s;
}

// Splits of the keys (tokens: the most a row attends to): the least rounds x (tiles a split + what a work-group costs besides).
inline int chunk_splits(const ChunkSizes& s, long long tokens) {
  const long long tiles = ceil_div(tokens, (long long)s.form.tile * s.form.token_waves);
  long long best = 1, best_cost = -1;
  for (long long n = 1; n <= s.split_most && n <= tiles; ++n) {
    const long long rounds = ceil_div(s.heads * s.row_blocks * n, kChunkGroups);
    const long long cost = rounds * (ceil_div(tiles, n) + 3) + (n > 1 ? 2 : 0);
    if (best_cost < 0 || cost < best_cost) { best = n; best_cost = cost; }
  }
  return (int)best;
}

}  // namespace innerq

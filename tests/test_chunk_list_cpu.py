"""The list that work-groups of a ragged attention over several new tokens make from the sequences' counts (csrc/chunk_plan.h, whose
arithmetic the kernel calls), walked on the CPU over random batches: every (sequence, head, block of rows, range) is some work-group's exactly once,
no item lies beyond the launch, and none that leaves a partial result beyond the workspace."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

MAIN = r"""
#include <stdio.h>
#include <algorithm>
#include <cmath>
#include <random>
#include <vector>
#include "paper_2602_23200_amd/csrc/chunk_plan.h"
using namespace innerq;

static long long lists = 0, lengthened = 0, uncut = 0, mixed = 0, bad = 0;
static void fail(const char* why, int batch, int heads, int r, int t) {
  if (++bad <= 10) printf("%s: batch %d heads %d r %d chunk %d\n", why, batch, heads, r, t);
}

// One launch: rows above `from` and up to `to`.
static void walk(const std::vector<int>& n, const std::vector<int>& t, int heads, int r, int most_new, int from, int to, const ChunkForm& f, long long groups, float nudge) {
  const int batch = (int)n.size(), tile = f.tile * f.token_waves;
  std::vector<ChunkShare> share(batch);
  int longest = 1;
  float work = 0.f;
  for (int b = 0; b < batch; ++b) {
    share[b] = chunk_share(n[b], t[b], r, heads, from, to, f.rows(), tile);
    longest = std::max(longest, share[b].tiles);
    work += (float)share[b].units * (float)share[b].tiles;
    const int rows = t[b] * r;
    if ((rows > from && rows <= to) != (share[b].units > 0)) fail("rows of the other launch", batch, heads, r, most_new);
    if (share[b].units && (long long)share[b].units / heads * f.rows() < rows) fail("rows left out", batch, heads, r, most_new);
    if (share[b].units && (long long)share[b].tiles * tile < n[b] + t[b]) fail("tokens left out", batch, heads, r, most_new);
  }
  int length = chunk_first_length(work * nudge), turns = 0;
  long long items;
  for (;; length = chunk_next_length(length), ++turns) {
    items = 0;
    for (const ChunkShare& s : share) items += (long long)s.units * chunk_ranges(s.tiles, length);
    if (items > 0x7fffffff) fail("more ranges than 31 bits count", batch, heads, r, most_new);
    if (chunk_length_fits(length, longest, (int)items)) break;
    if (turns > 1000) { fail("no end", batch, heads, r, most_new); return; }
  }
  ++lists;
  lengthened += turns > 0;
  if (items > groups) fail("more items than work-groups", batch, heads, r, most_new);
  bool cut = false, whole = false;
  long long first = 0;
  std::vector<char> seen;
  for (int b = 0; b < batch; ++b) {
    if (!share[b].units) continue;
    const int splits = chunk_ranges(share[b].tiles, length), blocks = share[b].units / heads;
    (splits > 1 ? cut : whole) = true;
    if (splits < 1 || (long long)splits * length < share[b].tiles) fail("tiles left out", batch, heads, r, most_new);
    const int all = share[b].units * splits;
    seen.assign(all, 0);
    for (int at = 0; at < all; ++at) {
      const ChunkPlace p = chunk_place(at, share[b].units, heads, splits);
      if (p.h < 0 || p.h >= heads || p.row_block < 0 || p.row_block >= blocks || p.split < 0 || p.split >= splits) { fail("place", batch, heads, r, most_new); continue; }
      char& mark = seen[((long long)p.h * blocks + p.row_block) * splits + p.split];
      if (mark) fail("twice", batch, heads, r, most_new);
      mark = 1;
      if (splits > 1 && first + at >= kChunkListItems) fail("a partial result beyond the workspace", batch, heads, r, most_new);
      // (where the merge looks for it)
      if (((long long)p.h * blocks + p.row_block) * splits + p.split != at) fail("slot", batch, heads, r, most_new);
    }
    first += all;
  }
  if (cut && items > kChunkListItems) fail("ranges of more items than aimed at", batch, heads, r, most_new);
  uncut += !cut && items > kChunkListItems;
  mixed += cut && whole;
}

int main() {
  std::mt19937 rng(1);
  auto draw = [&](double lo, double hi) { return (int)std::exp(std::uniform_real_distribution<double>(std::log(lo), std::log(hi))(rng)); };
  const int some_heads[] = {1, 2, 8, 8, 16, 32, 64}, some_r[] = {1, 2, 4, 4, 8, 71};
  for (int turn = 0; turn < 6000; ++turn) {
    const int batch = draw(1, 257), heads = some_heads[rng() % 7], r = some_r[rng() % 6], most_new = draw(1, 5000), most_cached = draw(1, 1 << (10 + rng() % 15));
    std::vector<int> n(batch), t(batch);
    for (int b = 0; b < batch; ++b) {
      n[b] = rng() % 4 == 0 ? 0 : draw(1, most_cached + 1);
      t[b] = rng() % 5 == 0 ? 0 : std::min(most_new, draw(1, most_new + 1));
    }
    innerq_config_t c = {};
    c.batch = batch; c.n_kv_heads = heads; c.n_q_heads = heads * r; c.head_dim = 128; c.capacity_tokens = 1 << 24;
    if ((long long)most_new * c.n_q_heads * batch >= (1LL << 31)) continue;
    const ChunkList list = chunk_list(c, most_new);
    if (!list.some) for (int x : t) if (x * r > kChunkWaveRows) fail("no launch for these rows", batch, heads, r, most_new);
    for (const float nudge : {1.0f, 0.999f, 1.001f}) {     // (the sum's order is the wavefront's own)
      walk(n, t, heads, r, most_new, 0, kChunkWaveRows, kFewRows, list.few, nudge);
      if (list.some) walk(n, t, heads, r, most_new, kChunkWaveRows, 0x7fffffff, kSomeRows, list.some, nudge);
    }
  }
  // as much work as 31 bits of rows have over as many tokens as a call may name: lengths and ranges stay within 31 bits
  for (float work = 1.0f; work < 1e14f; work *= 1.7f) {
    const int length = chunk_first_length(work);
    if (length < kChunkListLeast || (length < work / kChunkListItems - 1 && length < 1 << 19)) fail("first length", 0, 0, 0, 0);
    for (const int tiles : {1, 1000, 1 << 19})
      if (chunk_ranges(tiles, length) < 1 || (long long)chunk_ranges(tiles, length) * length < tiles) fail("ranges of a long length", 0, 0, 0, length);
  }
  printf("%lld lists, %lld lengthened, %lld of more items than aimed at, %lld cut in part, %lld bad\n", lists, lengthened, uncut, mixed, bad);
  return bad || lengthened < 500 || uncut < 500 || mixed < 500;
}
"""


def test_every_item_is_found_once(tmp_path):
    compiler = shutil.which("g++")
    if not compiler:
        pytest.skip("no g++")
    source, program = tmp_path / "list.cc", tmp_path / "list"
    source.write_text(MAIN)
    subprocess.run([compiler, "-std=c++17", "-O2", "-I", ROOT, str(source), "-o", str(program)], check=True)
    run = subprocess.run([str(program)], stdout=subprocess.PIPE, text=True, timeout=100)
    print(run.stdout)
    assert run.returncode == 0, run.stdout

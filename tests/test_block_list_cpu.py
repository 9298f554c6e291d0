"""The launch plan of attention over the 8-bit cache (csrc/block_plan.h, whose arithmetic the kernels call), walked on the CPU over random
calls.  Ragged batches: every (sequence, head, block of rows, range) is some work-group's exactly once, no item lies beyond its list, and none that
leaves a partial result beyond the workspace."""
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
#include "paper_2602_23200_amd/csrc/block_plan.h"
using namespace innerq;

static long long lists = 0, lengthened = 0, uncut = 0, mixed = 0, bad = 0;
static void fail(const char* why, int batch, int heads, int r, int t) {
  if (++bad <= 10) printf("%s: batch %d heads %d r %d new %d\n", why, batch, heads, r, t);
}

// One list: rows above `from` and up to `to`.
static void walk(const std::vector<int>& n, const std::vector<int>& t, bool causal, int heads, int r, int most_new, int from, int to, const BlockForm& f, long long groups,
                 float nudge) {
  const int batch = (int)n.size(), round = block_list_items(f);
  if (groups % 8) fail("not a multiple of eight", batch, heads, r, most_new);
  std::vector<BlockShare> share(batch);
  int longest = 1;
  float work = 0.f;
  for (int b = 0; b < batch; ++b) {
    share[b] = block_share(n[b], t[b], causal, r, heads, from, to, f.rows);
    longest = std::max(longest, share[b].tiles);
    work += (float)share[b].units * (float)share[b].tiles;
    const int rows = t[b] * r;
    if ((rows > from && rows <= to) != (share[b].units > 0)) fail("rows of the other list", batch, heads, r, most_new);
    if (share[b].units && (long long)share[b].units / heads * f.rows < rows) fail("rows left out", batch, heads, r, most_new);
    if (share[b].units && (long long)share[b].tiles * kBlockTile < n[b] + (causal ? t[b] : 0)) fail("tokens left out", batch, heads, r, most_new);
  }
  int length = block_first_length(work * nudge, round), turns = 0;
  long long items;
  for (;; ++turns) {
    items = 0;
    for (const BlockShare& s : share) items += (long long)s.units * block_ranges(s.tiles, length);
    if (items > 0x7fffffff) fail("more ranges than 31 bits count", batch, heads, r, most_new);
    if (block_length_fits(length, longest, (int)items, round)) break;
    const int next = block_next_length(length, (int)items, round);
    if (next <= length || turns > 1000) { fail("no end", batch, heads, r, most_new); return; }
    length = next;
  }
  ++lists;
  lengthened += turns > 0;
  if (items > groups) fail("more items than work-groups", batch, heads, r, most_new);
  // every work-group's range, as it finds it
  const bool by_head = block_by_head(heads);
  const int scale = by_head ? 8 : 1;
  std::vector<char> taken(items, 0);
  for (long long x = 0; x < groups; ++x) {
    const int place = block_turn((int)x, (int)items, by_head);
    if (place < 0) continue;
    long long first = 0;
    for (int b = 0; b < batch; ++b) {
      const int splits = block_ranges(share[b].tiles, length), all = share[b].units * splits / scale;
      if (place >= first && place < first + all) {
        const int range = block_range((int)(place - first), (int)x, share[b].units, heads, splits, by_head);
        if (range < 0 || range >= share[b].units * splits) { fail("a range that is none", batch, heads, r, most_new); break; }
        char& mark = taken[first * scale + range];
        if (mark) fail("a range twice", batch, heads, r, most_new);
        mark = 1;
        break;
      }
      first += all;
    }
  }
  for (const char x : taken) if (!x) { fail("a range of no work-group", batch, heads, r, most_new); break; }
  bool cut = false, whole = false;
  long long first = 0;
  std::vector<char> seen;
  for (int b = 0; b < batch; ++b) {
    if (!share[b].units) continue;
    const int splits = block_ranges(share[b].tiles, length), blocks = share[b].units / heads;
    (splits > 1 ? cut : whole) = true;
    if (splits < 1 || (long long)splits * length < share[b].tiles) fail("tiles left out", batch, heads, r, most_new);
    const int all = share[b].units * splits;
    seen.assign(all, 0);
    for (int at = 0; at < all; ++at) {
      const BlockPlace p = block_place(at, share[b].units, heads, splits);
      if (p.h < 0 || p.h >= heads || p.row_block < 0 || p.row_block >= blocks || p.split < 0 || p.split >= splits) { fail("place", batch, heads, r, most_new); continue; }
      char& mark = seen[((long long)p.h * blocks + p.row_block) * splits + p.split];
      if (mark) fail("a place twice", batch, heads, r, most_new);
      mark = 1;
      if (splits > 1 && first + at >= round) fail("a partial result beyond the workspace", batch, heads, r, most_new);
      // (where the merge looks for it)
      if (((long long)p.h * splits + p.split) * blocks + p.row_block != at) fail("slot", batch, heads, r, most_new);
    }
    first += all;
  }
  if (cut && items > round) fail("ranges of more items than aimed at", batch, heads, r, most_new);
  uncut += !cut && items > round;
  mixed += cut && whole;
}

int main() {
  std::mt19937 rng(1);
  auto draw = [&](double lo, double hi) { return (int)std::exp(std::uniform_real_distribution<double>(std::log(lo), std::log(hi))(rng)); };
  const int some_heads[] = {1, 2, 3, 8, 8, 16, 32, 64}, some_r[] = {1, 2, 4, 4, 7, 8, 16};
  long long used = 0, wide = 0;
  for (int turn = 0; turn < 2500; ++turn) {
    const int batch = draw(1, 300), heads = some_heads[rng() % 8], r = some_r[rng() % 7], most_new = draw(1, 5000), most_cached = draw(1, 1 << (10 + rng() % 15));
    const bool causal = rng() % 2;
    innerq_block_config_t c = {};
    c.batch = batch; c.n_kv_heads = heads; c.n_q_heads = heads * r; c.head_dim = 128; c.capacity_tokens = 1 << 24; c.block = 32 << rng() % 2;
    if ((long long)most_new * c.n_q_heads * batch >= (1LL << 31)) continue;
    const size_t bytes = block_workspace_bytes(c, most_new);
    const long long bound = rng() % 2 ? 1 << 24 : most_cached + most_new;
    const BlockList list = block_list(c, most_new, bound);
    if (!list.use) continue;
    ++used;
    if (kBlockTableBytes + block_list_items(list.form) * block_slot_bytes(list.form.rows) +
            (list.many ? block_list_items(kBlockMany.form) * block_slot_bytes(kBlockMany.form.rows) : 0) > bytes) fail("workspace of a list", batch, heads, r, most_new);
    std::vector<int> n(batch), t(batch);
    for (int b = 0; b < batch; ++b) {
      n[b] = rng() % 4 == 0 ? 0 : draw(1, most_cached + 1);
      t[b] = rng() % 5 == 0 ? 0 : std::min(most_new, draw(1, most_new + 1));
    }
    for (int x : t) if (x * r > list.few_most && !list.many) fail("no list for these rows", batch, heads, r, most_new);
    if (list.many && list.form.rows != 32) fail("no kernel of both lists", batch, heads, r, most_new);
    wide += list.few_most > list.form.rows;
    for (const float nudge : {1.0f, 0.999f, 1.001f}) {     // (the sum's order is the wavefront's own)
      walk(n, t, causal, heads, r, most_new, 0, list.few_most, list.form, list.few, nudge);
      if (list.many) walk(n, t, causal, heads, r, most_new, list.few_most, 0x7fffffff, kBlockMany.form, list.many, nudge);
    }
  }
  // as much work as 31 bits of rows have over as many tokens as a call may name: lengths and ranges stay within 31 bits
  for (float work = 1.0f; work < 1e14f; work *= 1.7f)
    for (const int round : {256, 512}) {
      const int length = block_first_length(work, round);
      if (length < kBlockListLeast || (length < work / round - 1 && length < 1 << 20)) fail("first length", 0, 0, 0, 0);
      for (const int tiles : {1, 1000, 1 << 19})
        if (block_ranges(tiles, length) < 1 || (long long)block_ranges(tiles, length) * length < tiles) fail("ranges of a long length", 0, 0, 0, length);
    }
  printf("%lld calls with a list, %lld of them of blocks of few rows alone, %lld lists, %lld lengthened, %lld of more items than aimed at, %lld cut in part, %lld bad\n", used, wide, lists, lengthened,
         uncut, mixed, bad);
  return bad || used < 800 || wide < 80 || lengthened < 200 || uncut < 120 || mixed < 200;
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

"""The launch plan of attention over several new tokens (csrc/chunk_plan.h), compiled for the CPU and walked over batches, heads,
chunk sizes and lengths: every launch has to fit the workspace that a caller is told to bring."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

MAIN = r"""
#include <stdio.h>
#include "paper_2602_23200_amd/csrc/chunk_plan.h"
using namespace innerq;

int main() {
  const int batches[] = {1, 2, 3, 8, 31, 64, 255, 256, 257, 2000}, heads[] = {1, 2, 8, 32}, rs[] = {1, 3, 4, 8, 71};
  const long long chunks[] = {1, 2, 5, 8, 9, 32, 33, 100, 128, 129, 500, 2048, 5000}, caps[] = {64, 1280, 32768, 1 << 20};
  long long plans = 0, split = 0, bad = 0;
  for (int b : batches) for (int h : heads) for (int r : rs) for (long long t : chunks) for (long long cap : caps) {
    if (t > cap || (long long)b * h > 65535) continue;
    innerq_config_t c = {};
    c.batch = b; c.n_kv_heads = h; c.n_q_heads = h * r; c.head_dim = 128; c.capacity_tokens = cap;
    const long long room = (long long)chunk_workspace_bytes(c, t) - kChunkTableBytes;
    for (long long n = 0; n + t <= cap; n = n * 5 / 3 + 1) {
      const ChunkSizes s = chunk_sizes(c, t, n);
      const long long splits = chunk_splits(s, n + t), slots = s.heads * s.row_blocks * splits;
      const char* why = nullptr;
      if (splits < 1 || splits > s.split_most) why = "splits";
      if (splits > 1 && slots * (long long)chunk_slot_bytes(s.form) > room) why = "workspace";
      if (splits > 1 && slots > 2 * s.form.round) why = "more than two rounds of split work";
      if (s.rows <= 32 && s.form.row_waves != 1) why = "form of few rows";
      if (s.row_blocks * s.form.rows() < s.rows) why = "rows left out";
      ++plans;
      split += splits > 1;
      if (why && ++bad <= 10) printf("%s: batch %d heads %d r %d chunk %lld capacity %lld cached %lld\n", why, b, h, r, t, cap, n);
    }
    if (b <= kChunkListMost) {
      const ChunkList l = chunk_list(c, t);
      const char* why = nullptr;
      if (kChunkListItems * (long long)(chunk_slot_bytes(kFewRows) + (l.some ? chunk_slot_bytes(kSomeRows) : 0)) > room) why = "workspace of a list";
      if (l.few < (long long)b * h || l.few < kChunkListItems) why = "list of few rows";
      if (t * r > 32 && (l.some < kChunkListItems || l.some * 128 < (long long)b * h * t * r)) why = "list of more rows";
      if (why && ++bad <= 10) printf("%s: batch %d heads %d r %d chunk %lld capacity %lld\n", why, b, h, r, t, cap);
    }
  }
  printf("%lld plans, %lld split, %lld bad\n", plans, split, bad);
  return bad || split < plans / 20;
}
"""


def test_every_plan_fits_its_workspace(tmp_path):
    compiler = shutil.which("g++")
    if not compiler:
        pytest.skip("no g++")
    source, program = tmp_path / "plan.cc", tmp_path / "plan"
    source.write_text(MAIN)
    subprocess.run([compiler, "-std=c++17", "-O2", "-I", ROOT, str(source), "-o", str(program)], check=True)
    run = subprocess.run([str(program)], stdout=subprocess.PIPE, text=True)
    print(run.stdout)
    assert run.returncode == 0, run.stdout

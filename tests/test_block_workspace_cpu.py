"""A workspace of the 8-bit cache's attention for so many rows of a sequence also serves every call of fewer: a program makes one for its longest chunk."""
import os
import shutil
import subprocess

import pytest

from paper_2602_23200_amd import binding as iq

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("batch", [1, 3, 8, 48, 49, 64, 96, 97, 256, 257, 1000])
@pytest.mark.parametrize("kv_heads,r", [(1, 1), (8, 4), (8, 5), (32, 1), (2, 71), (4, 17)])
def test_never_more_for_fewer_rows(batch, kv_heads, r):
    cfg = iq.make_block_config(batch, kv_heads * r, kv_heads, capacity_tokens=1 << 15)
    rows = sorted({t + e for t in (2 ** i for i in range(15)) for e in (-1, 0, 1) if t + e > 0} | {16 * i // r for i in range(1, 40)} - {0})
    rows = [t for t in rows if t * r * kv_heads * batch < 1 << 31]                           # (more are refused)
    sizes = [iq.innerq_block_workspace_bytes(cfg, t) for t in rows]
    assert sizes[0] > 0 and sizes == sorted(sizes), [(t, a, b) for t, a, b in zip(rows[1:], sizes, sizes[1:]) if b < a]
    assert sizes[-1] <= 80 << 20


MAIN = r"""
#include <stdio.h>
#include "paper_2602_23200_amd/csrc/block_plan.h"
using namespace innerq;
int main() {
  long long plans = 0, split = 0, bad = 0;
  for (int batch : {257, 300, 511, 512, 513, 1000, 2000}) for (int heads : {1, 2, 3, 8}) for (int r : {1, 4, 71}) for (long long t : {1, 5, 9, 33, 40, 129, 500, 3000}) {
    innerq_block_config_t c = {};
    c.batch = batch; c.n_kv_heads = heads; c.n_q_heads = heads * r; c.head_dim = 128; c.capacity_tokens = 1 << 24; c.block = 32;
    if (block_both_kinds(c, t) != (t * r > 32)) { ++bad; continue; }
    if (block_list_of(c, t, false).use || block_list_of(c, t, true).use) ++bad;
    if (t * r <= 32) continue;
    const long long room = (long long)block_workspace_bytes(c, t) - kBlockTableBytes;
    for (long long n = 0; n < 1 << 24; n = n * 5 / 3 + 1) {
      const BlockPlan p = block_plan_both(c, t, n);
      ++plans;
      split += p.n_splits > 1;
      if (p.form.rows != 128 || p.row_blocks != (t * r + 127) / 128 || p.n_splits < 1 || (p.n_splits > 1 && (long long)batch * heads * p.row_blocks * p.n_splits *
          (long long)block_slot_bytes(128) > room)) ++bad;
    }
  }
  printf("%lld plans, %lld split, %lld bad\n", plans, split, bad);
  return bad || split < 100;
}
"""


def test_large_ragged_batches_fit_their_workspace(tmp_path):
    """Batches without a list, whose work-groups take the form of their own sequence."""
    compiler = shutil.which("g++")
    if not compiler:
        pytest.skip("no g++")
    source, program = tmp_path / "both.cc", tmp_path / "both"
    source.write_text(MAIN)
    subprocess.run([compiler, "-std=c++17", "-O2", "-I", ROOT, str(source), "-o", str(program)], check=True)
    run = subprocess.run([str(program)], stdout=subprocess.PIPE, text=True)
    assert run.returncode == 0, run.stdout

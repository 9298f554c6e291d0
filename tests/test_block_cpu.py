"""The cache in 8 bits with block scales without a GPU: sizes, what the calls refuse, the launch plan, and that the tests' tolerances tell right from
wrong."""
import ctypes as C
import os
import shutil
import subprocess

import numpy as np
import pytest

from paper_2602_23200_amd import binding as iq
from tests import block_reference as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
D = 128


def config(**kw):
    c = iq.make_block_config(2, 8, 2, type=iq.INT8, block=32, capacity_tokens=640)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def test_struct_layout():
    assert C.sizeof(iq.innerq_block_config_t) == 6 * 4 + 2 * 8 and iq.innerq_block_config_t.capacity_tokens.offset == 24
    assert C.sizeof(iq.innerq_block_cache_t) == 6 * 8 + 8 + 8 and iq.innerq_block_cache_t.page_table.offset == 56


@pytest.mark.parametrize("change,want", [
    (dict(batch=0), iq.E_ARG), (dict(n_q_heads=7), iq.E_ARG), (dict(n_kv_heads=0), iq.E_ARG), (dict(head_dim=0), iq.E_ARG),
    (dict(head_dim=64), iq.E_UNSUPPORTED), (dict(type=2), iq.E_ARG), (dict(type=-1), iq.E_ARG), (dict(block=0), iq.E_ARG),
    (dict(block=16), iq.E_UNSUPPORTED), (dict(block=128), iq.E_UNSUPPORTED), (dict(capacity_tokens=0), iq.E_ARG),
    (dict(capacity_tokens=96), iq.E_ARG), (dict(capacity_tokens=(1 << 24) + 64), iq.E_UNSUPPORTED), (dict(page_pool_pages=-1), iq.E_ARG),
    (dict(page_pool_pages=1 << 31), iq.E_ARG), (dict(batch=40000), iq.E_ARG),
    (dict(block=64), iq.OK), (dict(type=iq.E4M3), iq.OK), (dict(capacity_tokens=1 << 24), iq.OK), (dict(page_pool_pages=7), iq.OK)])
def test_configurations(change, want):
    c = config(**change)
    assert iq.innerq_block_validate_config(c) == want
    if want != iq.OK:
        assert iq.innerq_block_buffer_bytes(c, 0) == 0 and iq.innerq_block_workspace_bytes(c, 1) == 0
    assert iq.lib().innerq_block_validate_config(None) == iq.E_NULL


def test_buffer_bytes():
    c = config(block=64)
    assert [iq.innerq_block_buffer_bytes(c, i) for i in range(-1, 7)] == [0] + 2 * [4 * 640 * D, 4 * 640 // 64 * 4, 4 * 64 * D * 2] + [0]
    c.page_pool_pages = 5
    assert [iq.innerq_block_buffer_bytes(c, i) for i in range(3)] == [5 * 2 * 64 * D, 5 * 2 * 4, 4 * 64 * D * 2]
    assert iq.innerq_block_workspace_bytes(c, 0) == 0 and iq.innerq_block_workspace_bytes(c, -1) == 0
    assert iq.innerq_block_workspace_bytes(c, (1 << 24) + 1) == 0 and iq.innerq_block_workspace_bytes(c, 1) >= 256


class Call:
    """A call's arguments, good but for the device pointers (aligned, never followed: every call here is refused first)."""

    def __init__(self, name, **kw):
        self.L, self.cfg, self.name = iq.lib(), config(**kw), name
        self.cache = iq.innerq_block_cache_t()
        for n in iq.BLOCK_BUFFER_NAMES:
            setattr(self.cache, n, 4096)
        self.cache.n_tokens = 100
        s = iq.innerq_strides_t
        self.a = dict(k=4096, ks=s(64 * D * 2, 64 * D, D), v=4096, vs=s(64 * D * 2, 64 * D, D), q=4096, qs=s(64 * D * 8, 64 * D, D), t=4,
                      out=4096, os=s(64 * D * 8, 64 * D, D), fp32=0, ws=4096, bytes=1 << 40, n=4096, tn=4096, most=400, first=0, stream=None)

    def __call__(self, cfg=True, cache=True, **change):
        a = dict(self.a, **change)
        ref_ = {x: None if a[x] is None else C.byref(a[x]) for x in ("ks", "vs", "qs", "os")}
        kv = (a["k"], ref_["ks"], a["v"], ref_["vs"])
        end = (a["out"], ref_["os"], a["fp32"], a["ws"], a["bytes"], a["stream"])
        args = {"append": (*kv, a["t"], a["stream"]), "append_ragged": (a["n"], a["tn"], *kv, a["t"], a["stream"]),
                "read": (a["first"], a["t"], *kv, a["stream"]), "read_ragged": (a["n"], a["tn"], a["t"], *kv, a["stream"]),
                "attention": (*kv, a["q"], ref_["qs"], a["t"], *end),
                "attention_ragged": (a["n"], a["tn"], a["most"], *kv, a["q"], ref_["qs"], a["t"], *end),
                "cross_attention": (a["q"], ref_["qs"], a["t"], *end),
                "cross_attention_ragged": (a["n"], a["tn"], a["most"], a["q"], ref_["qs"], a["t"], *end)}[self.name]
        return getattr(self.L, "innerq_block_" + self.name)(C.byref(self.cfg) if cfg else None, C.byref(self.cache) if cache else None, *args)


ALL = ["append", "append_ragged", "read", "read_ragged", "attention", "attention_ragged", "cross_attention", "cross_attention_ragged"]


@pytest.mark.parametrize("name", ALL)
def test_refusals(name):
    c, s = Call(name), iq.innerq_strides_t
    ragged, attends, cross = name.endswith("ragged"), "attention" in name, "cross" in name
    assert c(cfg=False) == iq.E_NULL and c(cache=False) == iq.E_NULL
    assert c(t=-1) == iq.E_ARG
    for field in iq.BLOCK_BUFFER_NAMES:
        for bad, want in ((None, iq.E_NULL), (4104, iq.E_ALIGN)):
            setattr(c.cache, field, bad)
            assert c() == want, field
        setattr(c.cache, field, 4096)
    c.cfg.page_pool_pages = 3
    assert c() == iq.E_NULL                                # (no page table)
    c.cache.page_table = 4098
    assert c() == iq.E_ALIGN
    c.cfg.page_pool_pages, c.cache.page_table = 0, None
    if ragged:
        assert c(n=None) == iq.E_NULL and c(n=4098) == iq.E_ALIGN and c(tn=4097) == iq.E_ALIGN
        assert c(t=641) == iq.E_CAPACITY or cross
        if attends:
            assert c(most=-1) == iq.E_ARG and c(most=641) == iq.E_CAPACITY and (cross or c(most=0) == iq.E_ARG)
    else:
        for bad in (-1, 641):
            c.cache.n_tokens = bad
            assert c() == iq.E_ARG
        c.cache.n_tokens = 100
        if name in ("append", "attention"):
            assert c(t=541) == iq.E_CAPACITY
        if name == "read":
            assert c(first=-1) == iq.E_ARG and c(first=97) == iq.E_ARG and c(first=101, t=0) == iq.E_ARG and c(t=2 ** 62, first=50) == iq.E_ARG
    writes = [("out", "os", 8)] if attends else [("k", "ks", 2), ("v", "vs", 2)] if "read" in name else []
    reads = ([] if "read" in name else [] if cross else [("k", "ks"), ("v", "vs")]) + ([("q", "qs")] if attends else [])
    for p, st in reads + [w[:2] for w in writes]:
        if "read" not in name:
            assert c(**{p: None}) == iq.E_NULL
        assert c(**{st: None}) == iq.E_NULL and c(**{p: 4100}) == iq.E_ALIGN
        assert c(**{st: s(-D, 0, D)}) == iq.E_ARG and c(**{st: s(64 * D * 8, 64 * D, D + 4)}) == iq.E_ALIGN
    for p, st, heads in writes:
        assert c(**{st: s(64 * D * heads, 64 * D, 0)}) == iq.E_ARG                     # rows over each other
        assert c(**{st: s(64 * D * heads, 3 * D, D)}) == iq.E_ARG
        assert c(**{st: s(0, 64 * D, D)}) == iq.E_ARG
    if "read" in name:
        assert c(k=None, v=None) == iq.E_NULL
    if attends:
        assert c(ws=None) == iq.E_NULL and c(ws=4104) == iq.E_ALIGN
        assert c(bytes=iq.innerq_block_workspace_bytes(c.cfg, 4) - 1) == iq.E_WORKSPACE
        if cross:
            assert c(t=(1 << 24) + 1) == iq.E_UNSUPPORTED
    # nothing to do
    assert c(t=0, **({"first": 100} if name == "read" else {})) == iq.OK
    assert c.cache.n_tokens == 100


PLAN = r"""
#include <stdio.h>
#include "paper_2602_23200_amd/csrc/block_plan.h"
using namespace innerq;
int main() {
  const int batches[] = {1, 2, 3, 8, 31, 64, 255, 256, 257, 2000}, heads[] = {1, 2, 8, 32}, rs[] = {1, 3, 4, 8, 71};
  const long long chunks[] = {1, 2, 5, 8, 16, 17, 33, 100, 500, 2048, 5000}, caps[] = {64, 1280, 32768, 1 << 20};
  long long plans = 0, split = 0, bad = 0;
  for (int b : batches) for (int h : heads) for (int r : rs) for (long long t : chunks) for (long long cap : caps) {
    if (t > cap || (long long)b * h > 65535) continue;
    innerq_block_config_t c = {};
    c.batch = b; c.n_kv_heads = h; c.n_q_heads = h * r; c.head_dim = 128; c.capacity_tokens = cap; c.block = 32;
    const long long room = (long long)block_workspace_bytes(c, t) - kBlockTableBytes;
    for (long long n = 0; n <= cap; n = n * 5 / 3 + 1) {
      const BlockPlan p = block_plan(c, t, n, n % 3 ? 0.f : 0.5f * t);
      const long long rows = t * r, slots = (long long)b * h * p.row_blocks * p.n_splits;
      const char* why = nullptr;
      if (p.n_splits < 1 || p.n_splits > block_split_most(p.form, (long long)b * h, p.row_blocks) || !(p.us > 0.f)) why = "splits";
      if (p.n_splits > 1 && (slots * (long long)block_slot_bytes(p.form.rows) > room || p.n_splits > (n + kBlockTile - 1) / kBlockTile)) why = "workspace";
      if (p.row_blocks * p.form.rows < rows || (p.row_blocks - 1) * p.form.rows >= rows || !block_suits(p.form, rows)) why = "rows";
      if ((p.form.rows > kBlockFewRows ? 32 * p.form.waves != p.form.rows : p.form.waves != 4)) why = "a form that there is no kernel of";
      ++plans;
      split += p.n_splits > 1;
      if (why && ++bad <= 10) printf("%s: batch %d heads %d r %d chunk %lld capacity %lld cached %lld\n", why, b, h, r, t, cap, n);
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
    source.write_text(PLAN)
    subprocess.run([compiler, "-std=c++17", "-O2", "-I", ROOT, str(source), "-o", str(program)], check=True)
    run = subprocess.run([str(program)], stdout=subprocess.PIPE, text=True)
    assert run.returncode == 0, run.stdout


def test_layout_of_the_header():
    """Bytes in the store's order, against the header's words."""
    x = np.arange(64 * D).reshape(1, 64, D)
    keys, values = ref.key_tiles(x)[0], ref.value_tiles(x)[0]
    for tile in range(2):
        at = 0
        for a in range(2):
            for h in range(2):
                for g in range(4):
                    for c in range(16):
                        assert (keys[tile, at:at + 16] == (32 * tile + 16 * a + c) * D + 32 * g + 16 * h + np.arange(16)).all()
                        at += 16
        at = 0
        for q in range(4):
            for g in range(4):
                for c in range(16):
                    for m in range(2):
                        for i in range(2):
                            assert (values[tile, at:at + 4] == (32 * tile + 16 * i + 4 * g + np.arange(4)) * D + 32 * q + 2 * c + m).all()
                            at += 4


def test_floating_point_codes():
    """All numbers of the type are their own nearest ones, bytes and values agree, halves go to even."""
    numbers = [(-1) ** (b >> 7) * ((b & 7) / 8 * 2.0 ** -6 if b >> 3 & 15 == 0 else (1 + (b & 7) / 8) * 2.0 ** ((b >> 3 & 15) - 7))
               for b in range(256)]
    for b, x in enumerate(numbers):
        if b & 0x7f == 0x7f:
            continue                                       # (no number)
        assert ref.e4m3(x) == x and ref.e4m3_bytes(np.float64(np.copysign(x, -1 if b >> 7 else 1))) == b
    assert ref.e4m3([17.0, 19.0, 2.0 ** -10, 3 * 2.0 ** -10, 440.0, 448.0, -17.0]).tolist() == [16.0, 20.0, 0.0, 2.0 ** -8, 448.0, 448.0, -16.0]


@pytest.mark.parametrize("many", [False, True])
def test_the_bound_tells_a_wrong_result(many):
    """One token more or fewer, a block's scale that is its neighbour's, (few rows) operands in bfloat16 are beyond the bound; rounding that
    it counts is within."""
    rng = np.random.default_rng(4)
    n, t = 200, 3
    k, v = rng.standard_normal((2, 1, n + t, D)).astype(np.float16)
    K, V = ref.held(k, 32, False), ref.held(v, 32, False)
    q = rng.standard_normal((1, t, D)).astype(np.float16)
    want, bound = ref.attend(q, K, V, False, many, ref.causal(n, t))

    def over(K, V, hidden=ref.causal(n, t), keep=lambda p: p):
        s = np.where(hidden, -np.inf, q[0].astype(np.float64) @ K[0].T / np.sqrt(D))
        p = keep(np.exp(s - s.max(-1, keepdims=True)))
        return (np.abs(p @ V[0] / p.sum(-1, keepdims=True) - want[0]) / bound[0]).max()

    def bf16(x):
        return (x.astype(np.float32).view(np.uint32) + 0x8000 & 0xffff0000).view(np.float32).astype(np.float64)

    fp16 = lambda x: x.astype(np.float16).astype(np.float64)  # noqa: E731
    assert over(K, V) <= 1e-6
    assert over(K, V, keep=lambda p: fp16(p * 512)) <= 1.0 if many else over(K, V, keep=lambda p: fp16(p) + fp16(p - fp16(p))) <= 1.0
    assert over(K, V, hidden=np.arange(n + t)[None] > n + np.arange(t)[:, None] - 1) > 3
    assert over(K, V, hidden=(np.arange(n + t)[None] > n + np.arange(t)[:, None]) | (np.arange(n + t) == 31)) > 3
    wrong = V.copy()
    wrong[:, 32:64] *= np.abs(v[:, 64:96]).max() / np.abs(v[:, 32:64]).max()
    assert over(K, wrong) > 3
    assert many or (over(bf16(K), V) > 1.5 and over(K, bf16(V)) > 1.5)

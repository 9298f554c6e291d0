"""The integers of the 8-bit cache as fp16 times a power of two (csrc/block_plan.h, int_codes): every code, every power that a block of values can have, rounded
once, as the definition says.  What the fused operation does is its definition, in 64 bits, rounded to fp16."""
import os
import shutil
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

MAIN = r"""
#include <stdio.h>
#include "paper_2602_23200_amd/csrc/block_plan.h"
int main() {
  for (int x = -45; x <= 5; ++x) printf("%d %u %u\n", x, innerq::int_codes(x), innerq::int_codes_top(innerq::int_codes(x)));
}
"""


def test_every_code_times_every_power(tmp_path):
    compiler = shutil.which("g++")
    if not compiler:
        pytest.skip("no g++")
    source, program = tmp_path / "codes.cc", tmp_path / "codes"
    source.write_text(MAIN)
    subprocess.run([compiler, "-std=c++17", "-O2", "-I", ROOT, str(source), "-o", str(program)], check=True)
    lines = subprocess.run([str(program)], stdout=subprocess.PIPE, text=True, check=True).stdout.split("\n")[:-1]
    assert len(lines) == 51
    code = np.arange(-128, 128)
    byte = code.astype(np.int8).view(np.uint8) ^ 0x80
    for line in lines:
        x, both, top = (int(y) for y in line.split())
        factor, bias = (np.array([h], np.uint16).view(np.float16).astype(np.float64) for h in (both & 0xffff, both >> 16))
        under = (byte.astype(np.uint16) | (top & 0xff) << 8).astype(np.uint16).view(np.float16).astype(np.float64)
        got = (under * factor + bias).astype(np.float16)   # (exact before the rounding: 64 bits hold all of it)
        want = (code * 2.0 ** x).astype(np.float16)
        assert np.array_equal(got, want), x
        assert (np.abs(got.astype(np.float64) - code * 2.0 ** x) <= 2.0 ** -25).all(), x

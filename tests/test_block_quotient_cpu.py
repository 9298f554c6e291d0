"""The quotient of the 8-bit cache's quantiser (csrc/block_store.hip): the product with the rounded reciprocal, put right by its remainder, is the
correctly rounded quotient for every fp16 value in a block whose largest magnitude is any fp16 number: all pairs, of either type.  (Signs change nothing; zeros are left to the tests on the device.)"""
import shutil
import subprocess

import pytest

MAIN = r"""
#include <math.h>
#include <cstdint>
#include <cstdio>
#include <thread>
#include <vector>
static float half(int h) { int e = h >> 10 & 31, m = h & 1023; return e ? ldexp((float)(1024 + m), e - 25) : ldexp((float)m, -24); }
int main() {
  std::vector<float> v;
  for (int i = 1; i < 0x7c00; ++i) v.push_back(half(i));
  long long bad[8] = {}, pairs[8] = {};
  for (float top : {127.f, 448.f}) {
    std::vector<std::thread> threads;
    for (int k = 0; k < 8; ++k) threads.emplace_back([&, k] {
      long long wrong = 0;
      for (size_t i = k; i < v.size(); i += 8) {
        const float s = v[i] / top, r = 1.0f / s;
        for (size_t j = 0; j <= i; ++j) {
          const float x = v[j], q = x * r;
          wrong += fmaf(-fmaf(q, s, -x), r, q) != x / s;
        }
        pairs[k] += i + 1;
      }
      bad[k] += wrong;
    });
    for (auto& t : threads) t.join();
  }
  long long all = 0, wrong = 0;
  for (int k = 0; k < 8; ++k) { all += pairs[k]; wrong += bad[k]; }
  printf("%lld pairs, %lld wrong\n", all, wrong);
  return wrong != 0 || all != 2 * (31743LL * 31744 / 2);
}
"""


def test_every_pair(tmp_path):
    compiler = shutil.which("g++")
    if not compiler or "avx2" not in open("/proc/cpuinfo").read():
        pytest.skip("no g++, or no fused multiply-add here")
    source, program = tmp_path / "quotient.cc", tmp_path / "quotient"
    source.write_text(MAIN)
    subprocess.run([compiler, "-std=c++17", "-O3", "-mavx2", "-mfma", "-ffp-contract=off", str(source), "-o", str(program), "-lpthread"], check=True)
    run = subprocess.run([str(program)], stdout=subprocess.PIPE, text=True)
    assert run.returncode == 0, run.stdout

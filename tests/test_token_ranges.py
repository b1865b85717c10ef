"""The tokens that a workgroup of an append or a read over tokens takes (csrc/kernels.hpp), on the CPU: every position of a request
once, also the last ones that 32 bits can number."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = r"""
#include "kernels.hpp"
#include <cstdio>
#include <initializer_list>
using namespace ellm;
int main() {
  int64_t wrong = 0, blocks = 0;
  const int64_t end = 0x7fffffff;
  auto check = [&](int64_t pos0, int64_t n) {
    if (pos0 < 0 || n < 1 || pos0 + n > end) return;
    int64_t at = pos0;
    const int32_t k = token_blocks(pos0, n);
    for (int32_t b = 0; b < k; b++, blocks++) {
      const TokenRange r = token_range((int32_t)pos0, (int32_t)n, b);
      const int64_t rows = (int64_t)r.p1 - r.p0;
      if (r.p0 != at || rows < 1 || rows > TOKEN_BLOCK || r.p0 / TOKEN_BLOCK != (r.p1 - 1) / TOKEN_BLOCK) wrong++;
      at = r.p1;
    }
    if (at != pos0 + n) wrong++;
  };
  for (int64_t from : {int64_t(0), int64_t(1000), int64_t(1) << 30, end - 200})
    for (int64_t pos0 = from; pos0 < from + 200; pos0++)
      for (int64_t n = 1; n < 200; n++) check(pos0, n);
  check(0, 1 << 20);
  check(end - (1 << 20), 1 << 20);
  std::printf("%lld %lld\n", (long long)wrong, (long long)blocks);
}
"""


def test_every_position_once(tmp_path):
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    if not os.path.exists(os.path.join(rocm, "include", "hip", "hip_runtime_api.h")):
        pytest.skip("no HIP headers")
    src, exe = tmp_path / "t.cpp", tmp_path / "t"
    src.write_text(PROGRAM)
    # (-fwrapv: what overflows wraps, as it does on the GPU)
    subprocess.run(["g++", "-O2", "-fwrapv", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(rocm, "include"),
                    "-I", os.path.join(ROOT, "paper_2506_15155_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    wrong, blocks = map(int, subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split())
    assert wrong == 0 and blocks > 100_000

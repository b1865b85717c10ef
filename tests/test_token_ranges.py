"""The tokens that a workgroup of an append or a read over tokens takes (csrc/kernels.hpp), on the CPU: every position of a request
once, also the last ones that 32 bits can number."""
import os
import subprocess

import pytest
import torch  # noqa: F401  (ahead of the package: both then use one HIP runtime, which the tests after this one need)

import paper_2506_15155_amd as E

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


def test_the_fused_append_refuses_what_the_append_refuses():
    """Tensors of 4-bit rows hold less than 2^31 tokens, whichever call brings the last one, and whatever the call's other tensors get."""
    cb = 1 << 31
    p = E.ellm_pool_create(None, None, cb, 1, 1, 64, 2, 400, flags=E.ELLM_POOL_METADATA_ONLY, device_bytes=800 * cb, dtype=E.ELLM_MXFP4)
    T = E.ellm_pool_get_geometry(p)["tokens_per_chunk"]
    t, other = E.ellm_tensor_create(p, 3 << 30), E.ellm_tensor_create(p, 2 * T)
    E.ellm_tensor_map_chunks(p, t, 0, -(-(3 << 30) // T))
    E.ellm_tensor_map_chunks(p, other, 0, 2)
    append = lambda ids, n: E.ellm_kv_append(p, ids, 16, 16, n, check=False)  # noqa: E731
    fused = lambda ids: E.ellm_kv_append_decode(p, ids, 16, 16, 16, 16, check=False)  # noqa: E731
    length = lambda x: E.ellm_tensor_get_table(p, x)[1]  # noqa: E731
    assert append([t], [(1 << 30) - 1]) == append([t], [(1 << 30) - 1]) == 0
    # 2^31 - 2 tokens: one more is taken, whether others come with it or not
    assert fused([other, t]) == E.ERR.NO_DEVICE
    assert append([t, other], [1, 500]) == 0 and length(t) == (1 << 31) - 1 and length(other) == 500
    assert append([other, t], [1, 1]) == fused([t]) == fused([other, t]) == E.ERR.RANGE and "2^31" in E.ellm_last_error()
    assert fused([other]) == E.ERR.NO_DEVICE
    assert length(t) == (1 << 31) - 1 and length(other) == 500
    E.ellm_pool_destroy(p)

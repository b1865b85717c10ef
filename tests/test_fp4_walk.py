"""Which rows the decode kernels over 4-bit rows ask for, tile by tile (csrc/fp4_walk.hpp), walked on the CPU: every token of a batch
once, no row outside its chunk, no table entry past a request's own, and nothing at all for the tile behind a share's last one,
whose loads the kernels issue as well."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = r"""
#include "fp4_walk.hpp"
#include <cstdio>
#include <random>
#include <vector>
using namespace ellm;
int64_t wrong = 0, tiles = 0, ends = 0;
void check(bool ok, const char* what, int32_t Tc, int32_t len) {
  if (!ok && wrong++ < 5) std::printf("%s: chunks of %d tokens, request of %d\n", what, Tc, len);
}
struct Tensor {
  const char* base;
  int32_t id, slots;
  uint32_t chunk(int32_t slot) const {
    check(slot >= 0 && slot < slots, "slot past the request's last", slot, slots);
    return (uint32_t)(id << 16 | slot);
  }
};
// the launch's waves (NW > 0: workgroups of NW waves, a step each) over requests of lens tokens
template <int U, bool RUN, bool APPEND, int NW>
void walk(const std::vector<int32_t>& lens, int32_t Tc, int32_t step_units, int64_t waves) {
  PoolView pv = {};
  pv.tokens_per_chunk = Tc;
  pv.units_per_chunk = (Tc + UNIT_TOKENS - 1) / UNIT_TOKENS;
  pv.by_chunk = divisor(Tc);
  pv.by_units = divisor(pv.units_per_chunk);
  BatchArgs a;
  a.n_req = (int32_t)lens.size();
  a.step_units = step_units;
  int64_t total = 0;
  std::vector<std::vector<int>> seen;
  for (int32_t i = 0; i < a.n_req; i++) {
    a.req[i] = {lens[i], i, (int32_t)total, 0, 1, 0};
    total += (units_of(lens[i], pv, pv.units_per_chunk) + step_units - 1) / step_units;
    seen.push_back(std::vector<int>(lens[i]));
  }
  if (NW || step_units > 1) waves = total;
  waves = std::min(waves, total);
  const int64_t each = total / waves, more = total % waves;
  auto open = [&](int32_t id) { return Tensor{nullptr, id, (lens[id] + Tc - 1) / Tc}; };
  for (int64_t w = 0; w < waves; w++) {
    const int32_t u_lo = (int32_t)(w * each + std::min(w, more)), n_units = (int32_t)(each + (w < more));
    int32_t b = 0;
    while (b + 1 < a.n_req && a.req[b + 1].unit_prefix <= u_lo) b++;
    for (int wave = 0; wave < (NW ? NW : 1); wave++) {
      Fp4Cursor<U, RUN, Tensor> cursor;
      cursor.template begin<NW>(pv, a, a.req[b], b, (int32_t)w, u_lo, n_units, wave, open);
      if (NW && cursor.rem_share <= 0) continue;
      for (bool end = false, behind = false; !behind;) {
        Fp4Tile<U, RUN> t;
        behind = end;
        cursor.next(pv, a, open, t);
        tiles++;
        check(behind == (t.n == 0), "a tile of no units that is not behind the last", Tc, lens[t.b]);
        int32_t unit = 0;
        for (int i = 0; i < t.PIECES; i++) {
          const int32_t n = t.template there<APPEND>(i);
          check(n >= 0 && t.r[i] >= 0 && t.r[i] + n <= Tc && t.r[i] < Tc, "rows outside their chunk", Tc, lens[t.b]);
          check(!behind || n == 0, "rows behind the share's last tile", Tc, lens[t.b]);
          check(n <= t.rows[i] && t.rows[i] <= (RUN ? U : 1) * UNIT_TOKENS, "more rows than the tile has", Tc, lens[t.b]);
          const int32_t pos0 = (int32_t)(t.at[i] & 0xffff) * Tc + t.r[i];
          check((int32_t)(t.at[i] >> 16) == t.b, "another request's chunk", Tc, lens[t.b]);
          for (int32_t k = 0; k < t.rows[i]; k++)
            if (pos0 + k < lens[t.b]) seen[t.b][pos0 + k]++;
            else check(false, "a row behind the request's last", Tc, lens[t.b]);
          const bool new_here = t.rows[i] > n;       // the row that a fused append puts there: the request's last one
          check(!new_here || (t.rows[i] == n + 1 && pos0 + n == lens[t.b] - 1 && n + 1 == (RUN ? t.rows[0] : t.tail)), "another row than the new one", Tc, lens[t.b]);
          if (new_here) ends++;
          unit += t.rows[i] > 0;
        }
        check(RUN || unit == t.n, "units without rows", Tc, lens[t.b]);
        end |= (t.flags & T_FIN) != 0 || NW > 0;
        if (NW) break;                               // (a wave of a block asks for one tile)
      }
    }
  }
  for (int32_t i = 0; i < a.n_req; i++)
    for (int n : seen[i]) check(n == 1, "a token read not once", Tc, lens[i]);
}
template <int U, bool RUN, bool APPEND>
void all(const std::vector<int32_t>& lens, int32_t Tc, std::mt19937& rng) {
  int64_t total = 0;
  for (int32_t n : lens) total += (n + 15) / 16;
  for (int64_t waves : {int64_t(1), int64_t(2), int64_t(3), int64_t(1 + rng() % 40), total / 2 + 1, total * 2}) walk<U, RUN, APPEND, 0>(lens, Tc, 1, waves);
  walk<U, RUN, APPEND, 0>(lens, Tc, STEP_UNITS, 0);
  if constexpr (!RUN) {
    if constexpr (U == 2) walk<2, false, APPEND, 8>(lens, Tc, BLOCK_UNITS, 0);
    else for (int32_t b = BLOCK_UNITS + 1; b <= WIDE_UNITS; b++) walk<WIDE_UNITS / WIDE_WAVES, false, APPEND, WIDE_WAVES>(lens, Tc, b, 0);
  }
}
int main() {
  std::mt19937 rng(1);
  for (int32_t Tc : {1, 5, 16, 24, 100, 255, 256, 272, 1024, 1920})
    for (int turn = 0; turn < 60; turn++) {
      std::vector<int32_t> lens(1 + rng() % 6);
      // lengths around whole units and chunks as often as others
      for (int32_t& n : lens) {
        const int32_t near = rng() % 3 == 0 ? Tc * (int32_t)(1 + rng() % 3) : rng() % 2 ? 16 * (int32_t)(1 + rng() % 40) : (int32_t)(1 + rng() % 900);
        n = std::max(1, std::min(4000, near + (int32_t)(rng() % 5) - 2));
      }
      all<2, false, false>(lens, Tc, rng); all<4, false, false>(lens, Tc, rng);
      all<2, false, true>(lens, Tc, rng); all<4, false, true>(lens, Tc, rng);
      if (Tc >= 256) {                              // chunks that are walked in runs
        all<2, true, false>(lens, Tc, rng); all<4, true, false>(lens, Tc, rng);
        all<2, true, true>(lens, Tc, rng); all<4, true, true>(lens, Tc, rng);
      }
    }
  std::printf("%lld %lld %lld\n", (long long)wrong, (long long)tiles, (long long)ends);
}
"""


def test_tiles_stay_inside_their_chunks(tmp_path):
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    if not os.path.exists(os.path.join(rocm, "include", "hip", "hip_runtime_api.h")):
        pytest.skip("no HIP headers")
    src, exe = tmp_path / "walk.cpp", tmp_path / "walk"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-O1", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(rocm, "include"),
                    "-I", os.path.join(ROOT, "paper_2506_15155_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout
    wrong, tiles, ends = map(int, out.splitlines()[-1].split())
    assert wrong == 0, out
    assert tiles > 100_000 and ends > 10_000

"""The tiles of the attention over 16-bit blocks, and stretches of calls that take them (CPU only: the plan is plain C++)."""
import os
import subprocess

import pytest

from tests import test_attend_plan

CSRC = test_attend_plan.CSRC

# tests/test_attend_plan.py's walk of a call's stretches, with these tiles, and with calls large enough for all of them
CALL, SIZES, LAST = "max_q, window));", "R = (int)pick(1, 6);", "return cut > 1000"
STRETCHES = (test_attend_plan.PROGRAM
             .replace("trial < 1200", "trial < 700")
             .replace(CALL, "max_q, window, rc::kv_kernel));\n    ++tiles[s.rows / 64];")
             .replace(SIZES, "R = (int)pick(1, trial % 5 ? 6 : 70);")
             .replace("long cut = 0", "long tiles[4] = {0, 0, 0, 0}, cut = 0")
             .replace("E = pick(0, trial % 3 == 0 ? 600 : 40)", "E = pick(0, trial % 3 && trial % 5 ? 40 : 500)")
             .replace("pick(1, trial % 2 ? 3 : 70)", "pick(1, trial % 2 && trial % 5 ? 3 : trial % 5 ? 70 : 160)")
             .replace(LAST, 'std::printf("%ld calls of few rows, %ld of 64, %ld of 128, %ld of 192\\n", tiles[0], tiles[1], tiles[2], tiles[3]);\n'
                            "  for (long n : tiles) REQUIRE(n >= 20);\n  " + LAST))

CHOICE = r"""
#include <cstdio>
#include "rc_attend_plan.hpp"
static int rows(int64_t n, double pairs, int64_t steps) { return rc::kv_kernel(n, pairs, steps).rows; }
#define REQUIRE(x) do { if (!(x)) { std::printf("line %d: %s\n", __LINE__, #x); return 1; } } while (0)
int main() {
  REQUIRE(rows(1, 1e6, 1000) == 16 && rows(16, 1, 1) == 16 && rows(17, 1, 1) == 32 && rows(32, 1e6, 1000) == 32);
  REQUIRE(rows(33, 1e6, 1000) == 64 && rows(64, 1e6, 1000) == 64 && rows(65, 1e6, 1000) == 192);
  // few tiles of 128 with little work: 64 rows, up to 256 of them and 4096 steps
  REQUIRE(rows(128, 256, 16) == 64 && rows(128, 257, 1) == 128 && rows(128, 256, 17) == 128 && rows(128, 1, 4096) == 64 && rows(128, 1, 4097) == 128);
  REQUIRE(rows(129, 128, 16) == 64 && rows(129, 129, 1) == 128);
  // 192 from 49152 steps on
  REQUIRE(rows(128, 768, 64) == 128 && rows(128, 768, 65) == 192 && rows(129, 384, 64) == 128 && rows(129, 385, 64) == 192);
  // all tiles of a size go by the same units: parts of a cut item fit the places that the workspace has
  for (int64_t n : {1, 17, 33, 65, 4000})
    for (double pairs : {1.0, 300.0, 1e5})
      for (int64_t steps : {1, 60, 5000}) {
        const rc::AttendKernel k = rc::kv_kernel(n, pairs, steps);
        REQUIRE(k.least > k.free && k.unit % 32 == 0 && k.wgs % 8 == 0 && (k.rows == 16) == (k.wgs == 768) && (k.rows > 32) == (k.unit == 64));
      }
  return 0;
}
"""


@pytest.mark.parametrize("program", ["CHOICE", "STRETCHES"])
def test_tiles_and_stretches(program, tmp_path):
    src, exe = tmp_path / "plan.cpp", str(tmp_path / "plan")
    src.write_text(globals()[program])
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-Wall", "-fsanitize=undefined,address", "-fno-sanitize-recover=all", "-I", CSRC, "-o", exe, str(src)])
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    print(r.stdout)
    assert r.returncode == 0, f"{r.returncode}: {r.stdout}{r.stderr}"


def test_the_walk_is_of_these_tiles():
    for text in ("rc::kv_kernel));", "tiles[s.rows / 64]", "trial % 5 ? 6 : 70", "long tiles[4]", "REQUIRE(n >= 20)", "trial < 700", "40 : 500", "70 : 160"):
        assert STRETCHES.count(text) == 1, text

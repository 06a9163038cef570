"""The plan of an attention call at its limits (CPU only: the plan is plain C++)."""
import os
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2507_21433_amd", "csrc")

HEAD = r"""
#include <cstdio>
#include "rc_attend_plan.hpp"

static unsigned long long state = 88172645463325252ull;
static int64_t pick(int64_t lo, int64_t hi) {
  state ^= state << 13, state ^= state >> 7, state ^= state << 17;
  return lo + (int64_t)(state % (unsigned long long)(hi - lo + 1));
}
#define REQUIRE(x) do { if (!(x)) { std::printf("line %d: %s\n", __LINE__, #x); return 1; } } while (0)
"""


def run(tmp_path, body):
    src, exe = tmp_path / "plan.cpp", str(tmp_path / "plan")
    src.write_text(HEAD + "int main() {\n" + body + "\n}\n")
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-Wall", "-fsanitize=undefined,address", "-fno-sanitize-recover=all", "-I", CSRC,
                           "-o", exe, str(src)])
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, f"{r.returncode}: {r.stdout}{r.stderr}"


def test_items_that_see_nothing_have_no_tokens(tmp_path):
    """Also where a window lies behind the end of a short table: an item has a run of tokens exactly where one of its rows sees a token, and then
    its limits hold some."""
    run(tmp_path, r"""
  long empty = 0, behind = 0;
  for (int trial = 0; trial < 200000; ++trial) {
    const int T = pick(0, 1) ? 16 : 32, g = (int)pick(1, 9);
    const int64_t E = pick(0, 9), max_q = pick(1, trial % 2 ? 3 : 70), window = pick(0, 3) ? pick(1, 60) : 0;
    rc::AttendShape s;
    REQUIRE(rc::attend_shape(&s, 1, 1, E, T, 1, g, max_q, max_q, window));
    const rc::AttendRequest q = rc::attend_request(s, (int32_t)pick(-2, E * T + 100), 0, (int32_t)pick(0, max_q));
    for (int t = 0; t < q.tiles; ++t) {
      const rc::AttendItem i = rc::attend_item(s, q, t);
      bool sees = false;
      for (int n = t * s.rows; n < q.rows && n < (t + 1) * s.rows; ++n) {
        const int pos = q.ctx - q.len + n / g;
        for (int k = 0; k < E * T; ++k) sees = sees || (k <= pos && (!window || k > pos - window));
      }
      REQUIRE(sees == (i.pairs > 0) && (sees ? i.low_min < i.high_max : i.units == 1 && i.free == 0));
      empty += !sees;
      behind += !sees && q.ctx > E * T;
    }
  }
  std::printf("%ld empty, %ld behind the table\n", empty, behind);
  return empty > 1000 && behind > 1000 ? 0 : 3;
""")

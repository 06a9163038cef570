"""The plan of an attention call at its limits (CPU only: the plan is plain C++)."""
import os
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2507_21433_amd", "csrc")

HEAD = r"""
#include <cstdio>
#include <vector>
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


def test_one_long_step_beside_many_short_ones(tmp_path):
    """A chunk beside hundreds of decoding requests, in many layers: the line is as long as the query tokens make it, not as if every request had
    the longest step.  (Units of 64 tokens mean that it was not thought to be too long.)"""
    run(tmp_path, r"""
  rc::AttendShape s;
  REQUIRE(rc::attend_shape(&s, 64, 512, 4096, 16, 8, 64, 8192 + 511, 8192, 0) && s.unit == 64);
  REQUIRE(rc::attend_shape(&s, 64, 4096, 8192, 16, 8, 64, 8192 + 4095, 8192, 0));
  // ... and what is too much is refused as before
  REQUIRE(!rc::attend_shape(&s, 64, 4096, 8192, 16, 8, 64, 1 << 29, 8192, 0));
  // its workspace is enough for every step of as many requests
  const size_t room = rc::attend_largest_workspace(64, 4096, 8192, 16, 8, 64, 8192);
  for (const int64_t n_q : {1, 100, 4096, 12287, 100000}) {
    REQUIRE(!rc::attend_shape(&s, 64, 4096, 8192, 16, 8, 64, n_q, 8192, 0) || rc::attend_workspace(s) <= room);
    REQUIRE(rc::attend_shape(&s, 64, 4096, 8192, 16, 8, 64, n_q, 1, 0) && rc::attend_workspace(s) <= room);
  }
  return 0;
""")


def test_the_line_is_no_longer_than_planned(tmp_path):
    """Units of requests in any mixture, counted as a workgroup counts them: they fit into 32 bits where starts ascend, and where they do not,
    the line is the true one or none."""
    run(tmp_path, r"""
  long none = 0, plain = 0, wild = 0, taken = 0;
  for (int trial = 0; trial < 4000; ++trial) {
    const int T = pick(0, 1) ? 16 : 32, H = (int)pick(1, 16), g = (int)pick(1, 16);
    const int64_t L = pick(0, 2) ? pick(1, 4) : pick(1, 4000), R = pick(0, 2) ? pick(1, 40) : pick(1, 700), E = pick(0, 1) ? pick(0, 200) : pick(0, 90000);
    const int64_t longest = pick(0, 1) ? pick(1, 5) : pick(1, 4000);
    const bool ascending = pick(0, 3) != 0;
    std::vector<int32_t> start(R + 1, 0), ctx(R);
    for (int64_t r = 0; r < R; ++r) {
      start[r + 1] = start[r] + (int32_t)(pick(0, 9) ? pick(0, 2) : pick(0, longest));
      ctx[r] = (int32_t)pick(-5, E * T + 10);
    }
    const int64_t n_q = start[R] + pick(0, 1);
    if (!ascending)
      for (auto& x : start) x = pick(0, 1) ? (int32_t)n_q + 5 : -5;
    rc::AttendShape s;
    if (!rc::attend_shape(&s, L, R, E, T, H, H * g, n_q, pick(0, 1) ? longest : n_q, 0)) continue;
    ++taken;
    int32_t total = 0;
    int64_t exact = 0;
    for (int64_t r = 0; r < R; ++r) {
      const int32_t n = rc::attend_units(s, rc::attend_request(s, ctx[r], start[r], start[r + 1])) * H;
      total = rc::attend_sum(total, n);
      exact += n;
    }
    const int32_t line = rc::attend_line(s, total);
    REQUIRE(line < 1 << 30 && (line == 0 || line == exact * L));
    if (ascending)
      REQUIRE(line == exact * L && ++plain);
    else
      exact * L >= 1 << 30 ? ++none : ++wild;
    const int64_t share = rc::attend_share(s, line);
    REQUIRE(share * s.wgs < 0x7fffffff && share * s.wgs >= line);
  }
  std::printf("%ld taken, %ld plain, %ld wild, %ld none\n", taken, plain, wild, none);
  return plain > 1000 && wild > 100 && none > 10 ? 0 : 3;
""")


def test_tiles_of_64_rows_where_those_of_128_are_little_work(tmp_path):
    """What was measured on both sides of the rule (us beside it in the plan): rows, tiles of 128, steps of 64 tokens."""
    run(tmp_path, r"""
  struct { int64_t rows; double pairs; int64_t steps; int32_t tile; } cases[] = {
      {128, 128, 16, 64}, {128, 128, 31, 64}, {128, 64, 78, 64}, {128, 32, 187, 64}, {128, 16, 406, 64}, {128, 128, 62, 64},
      {128, 128, 78, 128}, {128, 128, 125, 128}, {128, 64, 250, 128}, {128, 16, 937, 128}, {2000, 8, 125, 128}, {2048, 16, 14, 128}};
  for (const auto& c : cases) REQUIRE(rc::attend_kernel(c.rows, c.pairs, c.steps).rows == c.tile);
  return 0;
""")

"""How the work of an attention call is cut into stretches (CPU only: the plan is plain C++): every cached token that a row sees lies in its
item's units, the limits that let a run of tokens go without a mask are right, and every item's parts find places of their own."""
import os
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2507_21433_amd", "csrc")

PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include <set>
#include <vector>
#include "rc_attend_plan.hpp"

static unsigned long long state = 88172645463325252ull;
static int64_t pick(int64_t lo, int64_t hi) {
  state ^= state << 13, state ^= state >> 7, state ^= state << 17;
  return lo + (int64_t)(state % (unsigned long long)(hi - lo + 1));
}
#define REQUIRE(x) do { if (!(x)) { std::printf("line %d: %s\n", __LINE__, #x); return 1; } } while (0)

int main() {
  long cut = 0, empty = 0, whole = 0;
  for (int trial = 0; trial < 1200; ++trial) {
    const int T = pick(0, 1) ? 16 : 32, H = (int)pick(1, 4), g = (int)pick(1, 9), L = (int)pick(1, 3), R = (int)pick(1, 6);
    const int64_t E = pick(0, trial % 3 == 0 ? 600 : 40), max_q = pick(1, trial % 2 ? 3 : 70), window = pick(0, 2) ? 0 : pick(1, 700);
    std::vector<int32_t> ctx(R), start(R + 1, 0);
    for (int r = 0; r < R; ++r) {
      ctx[r] = (int32_t)pick(-2, E * T + 20);
      start[r + 1] = start[r] + (int32_t)pick(0, max_q);
    }
    const int64_t n_q = start[R] + pick(0, 2);
    rc::AttendShape s;
    REQUIRE(rc::attend_shape(&s, L, R, E, T, H, H * g, n_q, max_q, window));
    if (n_q == 0) continue;
    REQUIRE(s.unit % 128 == 0 || (s.rows >= 64 && s.unit % 64 == 0));
    std::vector<int64_t> before(R + 1, 0);
    std::vector<rc::AttendRequest> q(R);
    for (int r = 0; r < R; ++r) {
      q[r] = rc::attend_request(s, ctx[r], start[r], start[r + 1]);
      REQUIRE(q[r].rows == (q[r].len < s.max_q ? q[r].len : s.max_q) * g);
      before[r + 1] = before[r] + H * rc::attend_units(s, q[r]);
      for (int t = 0; t < q[r].tiles; ++t) {
        const rc::AttendItem i = rc::attend_item(s, q[r], t);
        REQUIRE(i.units >= 1 && i.units <= rc::attend_most_units(s) && (i.free == s.free || !i.pairs));
        REQUIRE(rc::attend_run(s, i, 0) == i.pair0 && rc::attend_run(s, i, i.free) == i.pair0 && rc::attend_run(s, i, i.units) == i.pair0 + i.pairs);
        for (int u = i.free; u + 1 < i.units; ++u) REQUIRE(rc::attend_run(s, i, u + 1) - rc::attend_run(s, i, u) == s.unit / 32);
        if (q[r].tiles == 1) {
          const rc::AttendItem o = rc::attend_only_item(s, q[r]);
          REQUIRE(o.pair0 == i.pair0 && o.pairs == i.pairs && o.units == i.units && o.free == i.free && o.low_min == i.low_min && o.low_max == i.low_max &&
                  o.high_min == i.high_min && o.high_max == i.high_max);
        }
        int lowest = 1 << 30, highest = 0;
        for (int n = t * s.rows; n < q[r].rows && n < (t + 1) * s.rows; ++n) {
          const int pos = q[r].ctx - q[r].len + n / g;
          int lo = 1 << 30, hi = 0;
          for (int k = 0; k < E * T; ++k)
            if (k <= pos && (!window || k > pos - window)) lo = lo < k ? lo : k, hi = k + 1;
          if (hi) {
            REQUIRE(lo == rc::attend_low(s, pos) && hi == rc::attend_high(s, pos));
            lowest = lowest < lo ? lowest : lo, highest = highest > hi ? highest : hi;
            REQUIRE(i.low_max >= lo && i.high_min <= hi && i.low_min <= lo && i.high_max >= hi);
            REQUIRE(i.pair0 * 32 <= lo && (i.pair0 + i.pairs) * 32 >= hi);
          } else {
            // no unmasked run: nothing lies between the limits of a row that sees nothing
            REQUIRE(i.low_max >= i.high_min);
          }
        }
        if (highest == 0) ++empty;
        else REQUIRE((i.pair0 + i.pairs - 1) * 32 < highest && lowest - i.pair0 * 32 < 32);
        REQUIRE((int64_t)(i.pair0 + i.pairs) * 32 < (int64_t)s.cap + 32);
      }
    }
    // stretches, walked as a workgroup does: every run of tokens once, every part of a cut item in a place of its own, the first one's border
    // leads to the last, workgroups enough
    const int64_t line = before[R] * L, share = rc::attend_share(s, line);
    REQUIRE(share * s.wgs >= line && s.wgs % 8 == 0 && share > s.free);
    struct Run { int64_t item, wg, place; int first, last; };
    std::vector<Run> runs;
    std::vector<int64_t> border(s.wgs, -1);
    for (int64_t w = 0; w < s.wgs; ++w) {
      int64_t at = 0, item = 0;
      for (int l = 0; l < L; ++l)
        for (int r = 0; r < R; ++r)
          for (int h = 0; h < H; ++h)
            for (int t = 0; t < q[r].tiles; ++t, ++item) {
              const rc::AttendItem i = rc::attend_item(s, q[r], t);
              const int64_t begin = at, end = at + i.units, from = w * share, to = from + share;
              at = end;
              if (end <= from || begin >= to) continue;
              const int u0 = (int)(from > begin ? from - begin : 0), u1 = (int)((to < end ? to : end) - begin);
              if (u1 <= i.free) continue;
              const bool first = u0 <= i.free, last = u1 == i.units;
              runs.push_back({item, w, first && last ? -1 : rc::attend_place(w, begin + u0 == from), rc::attend_run(s, i, u0), rc::attend_run(s, i, u1)});
              if (first && !last) border[w] = w + (i.units - u1 + share - 1) / share;
            }
    }
    std::vector<std::vector<Run>> by_item;
    int64_t items = 0;
    for (int r = 0; r < R; ++r) items += (int64_t)L * H * q[r].tiles;
    by_item.resize(items);
    for (const Run& x : runs) by_item[x.item].push_back(x);
    std::set<int64_t> places;
    int64_t item = 0;
    for (int l = 0; l < L; ++l)
      for (int r = 0; r < R; ++r)
        for (int h = 0; h < H; ++h)
          for (int t = 0; t < q[r].tiles; ++t, ++item) {
            const rc::AttendItem i = rc::attend_item(s, q[r], t);
            const std::vector<Run>& x = by_item[item];
            REQUIRE(!x.empty() && x.front().first == i.pair0 && x.back().last == i.pair0 + i.pairs);
            for (size_t k = 1; k < x.size(); ++k) REQUIRE(x[k].first == x[k - 1].last && x[k].last > x[k].first && x[k].wg == x[k - 1].wg + 1);
            if (x.size() == 1) {
              REQUIRE(x[0].place == -1);
              ++whole;
              continue;
            }
            REQUIRE(border[x[0].wg] == x.back().wg);
            for (const Run& y : x) {
              REQUIRE(y.place >= 0 && y.place < rc::attend_most_parts(s) && places.insert(y.place).second);
              // what the joining launch takes for the places: the border's own, and the stretches' first ones behind it
              if (y.wg != x[0].wg) REQUIRE(y.place == rc::attend_place(y.wg, true));
              ++cut;
            }
          }
  }
  std::printf("%ld parts, %ld whole, %ld empty\n", cut, whole, empty);
  rc::AttendShape s;
  REQUIRE(!rc::attend_shape(&s, 1, 1, 1LL << 27, 16, 1, 1, 1, 1, 0));
  REQUIRE(rc::attend_shape(&s, 1, 1, (1LL << 27) - 5, 16, 1, 1, 1, 1, 1LL << 40) && s.window == 0);
  REQUIRE(!rc::attend_shape(&s, 1, 1, 8, 16, 1, 64, 1LL << 29, 1LL << 29, 0));
  // a line of more than 2^30 units: longer ones, or none at all
  REQUIRE(rc::attend_shape(&s, 64, 4096, 8192, 16, 16, 16, 4096, 1, 0));
  REQUIRE(s.unit > 128 && s.unit % 128 == 0 && 64.0 * 4096 * 16 * rc::attend_most_units(s) <= (1 << 30));
  REQUIRE(!rc::attend_shape(&s, 65535, 4096, 8, 16, 16, 16, 4096, 1, 0));
  return cut > 1000 && whole > 1000 && empty > 100 ? 0 : 3;
}
"""


def test_stretches_cover_what_the_rows_see(tmp_path):
    src, exe = tmp_path / "plan.cpp", str(tmp_path / "plan")
    src.write_text(PROGRAM)
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-Wall", "-fsanitize=undefined,address", "-fno-sanitize-recover=all", "-I", CSRC,
                           "-o", exe, str(src)])
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, f"{r.returncode}: {r.stdout}{r.stderr}"

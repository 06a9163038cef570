"""How the lanes of a wave share the counting of requests' row tiles (CPU only: the plan is plain C++)."""
import os
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2507_21433_amd", "csrc")


def test_lanes_that_count_row_tiles(tmp_path):
    """Of all powers of two the one with which a wave has counted all requests' tiles in the fewest turns; every tile is counted once."""
    src, exe = tmp_path / "lanes.cpp", str(tmp_path / "lanes")
    src.write_text(r"""
#include <cstdio>
#include <vector>
#include "rc_attend_plan.hpp"
#define REQUIRE(x) do { if (!(x)) { std::printf("line %d: %s\n", __LINE__, #x); return 1; } } while (0)
int main() {
  for (long R : {0, 1, 2, 3, 7, 31, 32, 33, 64, 65, 200, 1000})
    for (long tiles : {0, 1, 2, 5, 16, 40, 157, 1000}) {
      const int n = rc::attend_lanes(R, tiles);
      REQUIRE(n >= 1 && n <= 64 && (n & (n - 1)) == 0);
      const auto turns = [&](long k) { return (R * k + 63) / 64 * ((tiles + k - 1) / k); };
      for (int k = 1; k <= 64; k *= 2) REQUIRE(turns(n) <= turns(k));
      // as the kernels walk: lane i takes tiles i % n, i % n + n, ... of the requests of group i / n
      std::vector<int> seen(R * tiles);
      const long each = (R + 64 / n - 1) / (64 / n);
      for (int lane = 0; lane < 64; ++lane)
        for (long i = 0; i < each; ++i) {
          const long r = lane / n * each + i;
          for (long t = lane % n; r < R && t < tiles; t += n) ++seen[r * tiles + t];
        }
      for (int s : seen) REQUIRE(s == 1);
    }
  return 0;
}
""")
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-Wall", "-I", CSRC, "-o", exe, str(src)])
    r = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout

"""Attention over 16-bit blocks where scores are minus infinity: such a token has a probability of 0, and a row that has no other is one that sees
nothing.  Needs a real MI355X."""
import math

import pytest
import torch

from tests.test_gpu_kv import BF, DEV, HALF, WIDE, Problem, say

pytestmark = pytest.mark.gpu
ROWS = [(1, 1, None), (1, 5, WIDE), (5, 3, None), (4, 8, None), (40, 2, None), (40, 2, WIDE), (150, 3, None)]


def problem(m, g, E, dtype):
    p = Problem([(300, m), (320, m), (333, m)], 2, g, 16, dtype, E=E, gathered=True)
    p.q[..., 3] = p.q[..., 3].abs() + 0.25           # a key of minus infinity there makes scores of minus infinity
    return p


@pytest.mark.parametrize("dtype", [HALF, BF])
@pytest.mark.parametrize("m,g,E", ROWS)
@pytest.mark.parametrize("window", [0, 200])
def test_blocks_scored_minus_infinity_are_as_if_they_were_not_there(m, g, E, dtype, window):
    say(m, g, E, dtype, window)
    p = problem(m, g, E, dtype)
    p.window = window
    for e in (0, 7, 8, 9, 10, 17):                   # blocks of the first request, two runs of 32 tokens among them; all of the second
        p.k[0, 16 * e:16 * e + 16, :, 3] = -math.inf
    p.k[0, 300:620, :, 3] = -math.inf
    p.rewrite()
    r = p.run()
    # the definition of the same without these blocks
    p.tables[0, 0, [0, 7, 8, 9, 10, 17]] = -1
    p.tables[0, 1] = -1
    p.check(r)
    assert not r["out"][0, m:2 * m].any() and (r["lse"][0, m:2 * m] == -math.inf).all()
    assert torch.equal(r["weights"][0, 1], p.gathered[0, 1]) and torch.isfinite(r["weights"]).all()


@pytest.mark.parametrize("dtype", [HALF, BF])
@pytest.mark.parametrize("m,g,E", ROWS)
def test_a_token_scored_minus_infinity_weighs_nothing(m, g, E, dtype):
    # a score of -0.25 * 60000 * 128^-0.5 = -1326 is a probability of 0 in fp32, in the middle of what all rows see: the same bits
    say(m, g, E, dtype)
    p = problem(m, g, E, dtype)
    got = []
    for x in (-60000.0, -math.inf):
        p.k[0, 100, 1, 3] = p.k[0, 300 + 101, 0, 3] = x
        p.rewrite()
        got.append(p.run())
    assert all(torch.equal(got[0][x], got[1][x]) and torch.isfinite(got[0][x]).all() for x in got[0])

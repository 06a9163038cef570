"""The bound of cancelling outputs (tests/cache_cancelling.py) tells probabilities held as two 16-bit numbers from those rounded once.  CPU only."""
import pytest
import torch

from tests import cache_cancelling

HALF, BF = torch.float16, torch.bfloat16


def cut(x, dtype):
    """To the type's number next to 0."""
    y = x.to(dtype).double()
    step = torch.where(y > x, torch.tensor(-1, dtype=torch.int16), torch.tensor(0, dtype=torch.int16))
    return ((y.to(dtype).view(torch.int16) + step).view(dtype)).double()


@pytest.mark.parametrize("dtype", [HALF, BF])
@pytest.mark.parametrize("rows,n", [(1, 40), (4, 64), (5, 110), (16, 97), (16, 128)])
@pytest.mark.parametrize("seed", [1, 2])
def test_bound_tells_one_rounding_from_two_numbers(rows, n, dtype, seed):
    g = torch.Generator()
    g.manual_seed(seed)
    q, k, v = cache_cancelling.problem(rows, n, dtype, g)
    v = v.double()
    p = cache_cancelling.weights(q, k)
    limit = cache_cancelling.bound(p, v, dtype)
    # weights as a kernel has them: relative to a reference 7 below the largest score in powers of two
    w = torch.exp2((q.double()[:, None] * k.double()[None]) * 1.4426950408889634)
    w = w / w.amax(1, keepdim=True) * 2.0 ** 7
    exact = p @ v

    def off(held):
        out = ((held @ v) / w.sum(1, keepdim=True)).to(dtype).double()
        return (out - exact).abs() / limit

    for take in (cut, lambda x, dtype: x.to(dtype).double()):
        high = take(w, dtype)
        assert off(high + take(w - high, dtype)).max() <= 1
        assert off(high).max() > 1.5

"""The 4-bit cache and the attention over it at the limits of their types and arguments.  Needs a real MI355X."""
import math

import pytest
import torch

from paper_2507_21433_amd import binding as rc
from tests import cache_reference as ref
from tests.test_gpu_cache import BF, DEV, HALF, WIDE, Problem, gen, randn, say

pytestmark = pytest.mark.gpu

# query tokens, query heads of a KV head, entries of a table: tiles of 16, 32, 64 and 128 rows, items that are cut and whole ones
KERNELS = [(1, 4, None), (1, 4, WIDE), (5, 4, None), (5, 4, WIDE), (12, 4, None), (12, 4, WIDE), (40, 4, 20 * WIDE)]


def rewrite(p, k=None, v=None):
    """Other keys and values at a problem's tokens."""
    p.k, p.v = p.k if k is None else k.to(p.k.dtype), p.v if v is None else v.to(p.v.dtype)
    rc.rc_cache_write(p.k.to(DEV), p.v.to(DEV), p.slots.to(DEV), p.cache)


# ---- values as large as bf16 has them

@pytest.mark.parametrize("m,g,E", KERNELS)
@pytest.mark.parametrize("n,keys", [(1, "any"), (40, "any"), (700, "climbing"), (6000, "equal"), (70000, "equal")])
def test_largest_bf16_values(n, keys, m, g, E):
    """All tokens have the same values, up to 6 * 2^125: so has every weighted mean of them."""
    say(n, keys, m, g, E)
    p = Problem([(max(n, m), m), (m, m)], 1, g, 16, BF, E=E)
    v = torch.tensor([6.0, -4.0, 1.0, -6.0, 0.0, 3.0, -0.5, 2.0]).repeat(16) * 2.0 ** 125
    k = p.k.float()
    if keys == "equal":
        k = torch.zeros_like(k)
    elif keys == "climbing":
        k = torch.zeros_like(k)
        k[0, :n, 0, 0] = torch.arange(n) / 16.0
        p.q[..., 0] = 6.0
    rewrite(p, k, v.expand(p.v.shape))
    r = p.run()
    want = v.double().expand(r["out"].shape)
    # one rounding of the result, one of the probabilities where they are rounded once, sums and exponentials as in cache_reference.Bound
    h = torch.finfo(BF).eps / 2
    off = (r["out"].cpu().double() - want).abs()
    assert (off <= want.abs() * (h + (h if p.many else h * h) + 2.0 ** -11)).all(), off.max()
    assert torch.isfinite(r["lse"]).all()


@pytest.mark.parametrize("m,g,E", KERNELS)
@pytest.mark.parametrize("first", [0, 37, 300, 650])
def test_some_large_bf16_values(m, g, E, first):
    """Large values from some token on, in one of a token's groups, beside ordinary and small ones."""
    say(m, g, E, first)
    p = Problem([(700, m), (90, m)], 2, g, 16, BF, E=E, seed=first)
    gn = gen(first)
    v = p.v.float()
    large = torch.rand(v.shape[:3], generator=gn) < 0.1
    large[:, :first] = False
    v[..., 32:64] *= torch.where(large, 2.0 ** 124, 1.0)[..., None]
    v[..., 64:96] *= 2.0 ** -60
    rewrite(p, v=v)
    want, lse, bound = ref.attend(p.q, p.cache, p.tables, p.ctx, p.starts, p.scale, 0, p.many, tiny=2.0 ** -133)
    r = p.run()
    assert ((r["out"].cpu().double() - want).abs() <= bound.out).all()
    assert ((r["lse"].cpu().double() - lse).abs() <= bound.lse).all()


@pytest.mark.parametrize("m,g,E", KERNELS)
def test_smallest_bf16_values(m, g, E):
    """Values down to 0.5 * 2^-125 keep what the type has of them."""
    p = Problem([(200, m), (64, m)], 1, g, 16, BF, E=E, spread=2.0 ** -118)
    want, _, bound = ref.attend(p.q, p.cache, p.tables, p.ctx, p.starts, p.scale, 0, p.many, tiny=2.0 ** -133)
    assert ((p.run()["out"].cpu().double() - want).abs() <= bound.out).all()

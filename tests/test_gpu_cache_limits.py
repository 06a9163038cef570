"""The 4-bit cache and the attention over it at the limits of their types and arguments.  Needs a real MI355X."""
import math

import pytest
import torch

from paper_2507_21433_amd import binding as rc
from tests import cache_cancelling
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


# ---- scores as large as fp32 has them

def one_dim(p, k, q):
    """Keys and queries with a first dim only: scores are exact products."""
    keys = torch.zeros(p.k.shape)
    keys[..., 0] = k
    p.q.zero_()
    p.q[..., 0] = q.to(p.q.dtype).to(DEV)
    return keys


@pytest.mark.parametrize("m,g,E", KERNELS)
@pytest.mark.parametrize("dtype,large", [(HALF, False), (BF, False), (BF, True)])
@pytest.mark.parametrize("scale", [0.01, 3.0, 1e3, 1e6, 1e20])
def test_weights_of_huge_scores(m, g, E, dtype, large, scale):
    """Keys of a few levels far apart: a query's weights are shared equally by the tokens of the highest level that it sees."""
    say(m, g, E, dtype, large, scale)
    p = Problem([(500, m), (77, m)], 1, g, 16, dtype, E=E)
    gn = gen(int(m + min(scale, 2e6)))
    levels = torch.tensor([-6.0, -4.0, -2.0, 1.0, 3.0, 4.0, 6.0]) * 2.0 ** 10
    pick = torch.randint(0, 4, (500 + 77,), generator=gn)
    pick[130:] += torch.randint(0, 3, (500 + 77 - 130,), generator=gn)          # higher levels are met later
    pick[350:] += (torch.rand(500 + 77 - 350, generator=gn) < 0.05).int()
    q = (100 + 900 * torch.rand(p.q.shape[:3], generator=gn)) * torch.where(torch.rand(p.q.shape[:3], generator=gn) < 0.3, -1.0, 1.0)
    rewrite(p, one_dim(p, levels[pick][:, None].expand(p.k.shape[:3]), q), p.v.float() * 2.0 ** 123 if large else None)
    p.scale = scale
    r = p.run()
    values = ref.read(p.cache, torch.arange(p.cache.shape[1]))[1][0].reshape(-1, 128)
    h = torch.finfo(dtype).eps / 2
    for i, (n, new) in enumerate(zip(p.ctx, p.new)):
        at = p.slots[sum(p.ctx[:i]):][:n].long()
        for j in range(new):
            for a in range(g):
                x = levels[pick[sum(p.ctx[:i]):][:n - new + j + 1]].double() * p.q[0, p.starts[i] + j, a, 0].item()
                v = values[at[:x.numel()]][x == x.max()]
                got, lse = r["out"][0, p.starts[i] + j, a].cpu().double(), r["lse"][0, p.starts[i] + j, a].item()
                want, size = v.mean(0), v.abs().mean(0)
                off = (got - want).abs()
                assert (off <= h * want.abs() + ((h if p.many else h * h) + 2.0 ** -12) * size + (0 if dtype == BF else 2.0 ** -24)).all(), (i, j, a, off.max())
                # two roundings of the scale's product, one of the score's and one of the result
                exact = x.max().item() * scale + math.log(v.shape[0])
                assert abs(lse - exact) <= 2.0 ** -22 * abs(exact) + 2.0 ** -20


@pytest.mark.parametrize("m,g,E", KERNELS)
@pytest.mark.parametrize("dtype", [HALF, BF])
@pytest.mark.parametrize("scale", [1e6, 1e8, 1e9, 1e10])
def test_huge_scores_give_means(m, g, E, dtype, scale):
    """However coarse scores are, an output lies between the least and the largest of its values."""
    say(m, g, E, dtype, scale)
    p = Problem([(300, m), (40, m)], 2, g, 16, dtype, E=E, strong=True)
    p.scale = scale
    out = p.run()["out"].cpu().double()
    values = ref.read(p.cache, torch.arange(p.cache.shape[1]))[1][0].reshape(-1, 2, 128)
    h = torch.finfo(dtype).eps / 2
    for i, n in enumerate(p.ctx):
        at = p.slots[sum(p.ctx[:i]):][:n].long()
        for head in range(2 * g):
            v = values[at, head // g]
            got = out[0, p.starts[i]:p.starts[i + 1], head]
            room = 2 * (h + 2.0 ** -12) * v.abs().amax(0)
            assert (got >= v.amin(0) - room).all() and (got <= v.amax(0) + room).all()


# ---- windows behind the end of a table

@pytest.mark.parametrize("T,E,dtype", [(16, 3, HALF), (16, 13, BF), (32, 2, HALF), (16, 67, BF)])
@pytest.mark.parametrize("m,g", [(1, 4), (5, 4), (12, 4), (40, 4)])
def test_window_behind_a_short_table(T, E, dtype, m, g):
    """Queries whose window has slid past what the table lists see nothing, whatever its last block holds."""
    say(T, E, dtype, m, g)
    for past in (8, 9, 15, 16, 17, 40):
        p = Problem([(E * T + past + m - 1, m), (max(m, E * T - 3), m)], 1, g, T, dtype, E=E)
        p.window = 8
        last = p.tables[0, 0, E - 1].item()
        p.cache[0, last, ..., 2112:] = 254          # powers of V that become infinite
        p.cache[0, last, ..., 1024:2048] = 0x77
        r = p.run()
        assert (r["out"][0, :m] == 0).all() and (r["lse"][0, :m] == -math.inf).all(), past
        p.check(r)


# ---- memory that was never written

@pytest.mark.parametrize("m,g,E", KERNELS + [(20, 5, 20 * WIDE), (1, 5, None), (1, 3, WIDE), (7, 7, None)])
@pytest.mark.parametrize("dtype", [HALF, BF])
def test_unwritten_memory_leaves_no_trace(m, g, E, dtype):
    """Places behind the contexts, in blocks that the tables list, hold one thing or another: the results are the same bits."""
    say(m, g, E, dtype)
    p = Problem([(m + 37 * i, m) for i in range(24)], 2, g, 16, dtype, E=E)
    results = []
    for seed in (1, 2, 3):
        p.cache.copy_(torch.randint(0, 256, p.cache.shape, generator=gen(seed), dtype=torch.uint8))
        rewrite(p)
        results.append(p.run())
    for r in results[1:]:
        assert torch.equal(r["out"], results[0]["out"]) and torch.equal(r["lse"], results[0]["lse"])


# ---- many requests, long and short steps in one call

@pytest.mark.parametrize("R", [64, 65, 130, 200, 1000])
@pytest.mark.parametrize("m,g,E", [(1, 4, None), (1, 4, 100), (3, 8, 90), (9, 4, 90), (20, 4, None), (20, 4, 90)])
def test_many_requests(R, m, g, E):
    """More requests than a wave has lanes: tokens of all, of some, or of none, contexts from none to some hundreds."""
    say(R, m, g, E)
    gn = gen(R + m)
    new = torch.randint(0, 3, (R,), generator=gn).clamp(max=m).tolist()
    ctx = torch.randint(0, 90, (R,), generator=gn).tolist()
    for r in (3, R - 1, R // 2):
        new[r], ctx[r] = m, 90
    ctx[R // 3] = 1300 if E else 700
    p = Problem([(max(c, 0), n) for c, n in zip(ctx, new)], 2, g, 16, HALF, E=E)
    p.check(p.run())


@pytest.mark.parametrize("R,E,L", [(30, None, 1), (100, 100, 2)])
@pytest.mark.parametrize("dtype", [HALF, BF])
def test_a_chunk_beside_decoding_requests(R, E, L, dtype):
    say(R, E, L, dtype)
    gn = gen(R)
    requests = [(int(torch.randint(1, 250, (1,), generator=gn)), 1) for _ in range(R)]
    requests[R // 2] = (900, 150)
    p = Problem(requests, 2, 5, 16, dtype, L=L, E=E)
    p.check(p.run())


def test_starts_that_make_the_line_too_long():
    """Starts that go up and down would give every other request all query tokens: more units than there can be, and nothing is computed."""
    R, n_q, E, L, H = 6000, 64, 20000, 8, 16
    cache, dev = rc.cache_tensor(L, 1, 16, H, DEV), dict(dtype=torch.int32, device=DEV)
    starts = torch.zeros(R + 1, **dev)
    starts[1::2] = n_q
    assert L * (R // 2) * H * (E * 16 // 64) > 1 << 30
    q = torch.randn((L, n_q, H, 128), device=DEV).to(HALF)
    out, lse = torch.full_like(q, 7.0), torch.full((L, n_q, H), 7.0, device=DEV)
    rc.rc_cache_attend(q, cache, torch.zeros((L, R, E), **dev), torch.full((R,), E * 16, **dev), q_start=starts, max_q=n_q, out=out, lse=lse)
    torch.cuda.synchronize()
    assert (out == 7).all() and (lse == 7).all()


@pytest.mark.parametrize("requests", [[(30, 3), (20, 0), (20, 2)], [(400, 60), (90, 1), (5, 5)]])
def test_max_q_left_out(requests):
    """Without it every query token is computed."""
    p = Problem(requests, 2, 3, 16, HALF)
    i = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    out, lse = torch.full_like(p.q, 7.0), torch.full(p.q.shape[:3], 7.0, device=DEV)
    p.many = sum(p.new) * 3 > 16
    p.check(rc.rc_cache_attend(p.q, p.cache, p.tables.to(DEV), i(p.ctx), q_start=i(p.starts), out=out, lse=lse))


# ---- a cache of no blocks

@pytest.mark.parametrize("dtype", [HALF, BF])
def test_cache_of_no_blocks(dtype):
    """Nothing is stored, every block is read as zeros, nothing is seen."""
    i = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    cache = rc.cache_tensor(2, 0, 32, 3, DEV)
    kv = torch.ones((2, 4, 3, 128), dtype=dtype, device=DEV)
    rc.rc_cache_write(kv, kv, i([0, 5, -1, 31]), cache)
    k, v = (torch.full((2, 3, 32, 3, 128), 7.0, dtype=dtype, device=DEV) for _ in range(2))
    rc.rc_cache_read(cache, i([0, -1, 2]), k=k, v=v)
    assert not k.any() and not v.any()
    r = rc.rc_cache_attend(torch.ones((2, 2, 6, 128), dtype=dtype, device=DEV), cache, torch.zeros((2, 2, 50), dtype=torch.int32, device=DEV), i([40, 3]))
    assert not r["out"].any() and (r["lse"] == -math.inf).all()


# ---- probabilities of few rows

@pytest.mark.parametrize("dtype", [HALF, BF])
@pytest.mark.parametrize("g,n,E", [(1, 40, None), (4, 64, None), (5, 110, WIDE), (16, 97, None), (16, 128, WIDE)])
@pytest.mark.parametrize("seed", [1, 2])
def test_few_rows_lose_nothing_of_their_probabilities(g, n, E, dtype, seed):
    """With up to 16 rows a probability is the sum of two 16-bit numbers: outputs that nearly cancel are as close as that makes them."""
    say(g, n, E, dtype, seed)
    p = Problem([(n, 1)], 1, g, 16, dtype, E=E)
    q, k, v = cache_cancelling.problem(g, n, dtype, gen(seed))
    rewrite(p, one_dim(p, k.float()[:, None], q[None, None]), v.float()[None, :, None])
    held = [x[0].reshape(-1, 128)[p.slots.long()] for x in ref.read(p.cache, torch.arange(p.cache.shape[1]))]
    assert torch.equal(held[0][:, 0], k.double()) and torch.equal(held[1], v.double())
    p.scale = 1.0
    weights = cache_cancelling.weights(q, k)
    off = (p.run()["out"][0, 0].cpu().double() - weights @ v.double()).abs() / cache_cancelling.bound(weights, v.double(), dtype)
    say("largest error in bounds:", off.max().item())
    assert off.max() <= 1

"""16-bit blocks on the GPU: tokens stored into them, attention over them and what blocks gather within the bounds that the arithmetic allows, eviction
entry by entry as defined (tests/kv_reference.py).  Needs a real MI355X."""
import math
import sys

import pytest
import torch

from paper_2507_21433_amd import binding as rc
from tests import cache_cancelling
from tests import kv_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HALF, BF = torch.float16, torch.bfloat16


def say(*msg):
    print("[gpu-case]", *msg, flush=True)
    sys.stdout.flush()


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def randn(shape, g, dtype=torch.float32):
    return torch.randn(shape, generator=g, dtype=torch.float32).to(dtype)


def garbage(shape, dtype, g):
    """Any bits, infinities and NaNs among them: what memory holds that was never written."""
    return torch.randint(-32768, 32768, shape, generator=g, dtype=torch.int32).to(torch.int16).view(dtype)


def bits(x):
    return x.view(torch.int16)


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


# ---- write

@pytest.mark.parametrize("L,T,H,N,dtype", [(1, 16, 1, 1, HALF), (1, 16, 8, 3, BF), (3, 32, 5, 16, HALF), (2, 16, 16, 17, BF), (1, 32, 4, 33, BF),
                                           (2, 16, 10, 64, HALF), (1, 16, 3, 131, BF), (2, 32, 8, 96, HALF)])
@pytest.mark.parametrize("order", ["whole", "runs", "anywhere", "fused"])
def test_write(L, T, H, N, dtype, order):
    say(L, T, H, N, dtype, order)
    g = gen(N * 7 + H)
    NB = 2 * (N // T + 2)
    if order == "fused":
        wide = garbage((L, N, 4 * H, 128), dtype, g).to(DEV)
        k, v = wide[:, :, 2 * H:3 * H], wide[:, :, 3 * H:]
    else:
        k, v = garbage((L, N, H, 128), dtype, g).to(DEV), garbage((L, N, H, 128), dtype, g).to(DEV)
    if order == "whole":
        slots = torch.arange(N, dtype=torch.int32) + T
    elif order == "runs":
        slots = torch.arange(N, dtype=torch.int32) + 5
        slots[N // 2:] += 7
    else:
        slots = torch.randperm(NB * T, generator=g)[:N].to(torch.int32)
    if N > 2:
        slots[N // 3], slots[N - 1] = -1, NB * T     # neither is stored
    # a part of a larger pool: layers lie apart, blocks of others on both sides
    pools = [garbage((L, NB + 2, T, H, 128), dtype, g) for _ in range(2)]
    dev = [x.to(DEV) for x in pools]
    rc.rc_kv_write(k, v, slots.to(DEV), dev[0][:, 1:NB + 1], dev[1][:, 1:NB + 1])
    for pool, got, new in zip(pools, dev, (k, v)):
        want = pool.clone()
        want[:, 1:NB + 1] = ref.write(pool[:, 1:NB + 1], new.cpu(), slots)
        assert torch.equal(bits(got.cpu()), bits(want))


def test_nothing_to_write():
    k = torch.zeros((1, 4, 16, 2, 128), dtype=HALF, device=DEV)
    new = torch.ones((1, 0, 2, 128), dtype=HALF, device=DEV)
    rc.rc_kv_write(new, new, ints([]), k, k)
    none = torch.zeros((1, 0, 16, 2, 128), dtype=HALF, device=DEV)
    one = torch.ones((1, 1, 2, 128), dtype=HALF, device=DEV)
    rc.rc_kv_write(one, one, ints([0]), none, none)
    assert not k.any()


# ---- attend

class Problem:
    """Requests of (cached tokens, query tokens) over blocks that lie anywhere among unwritten ones."""

    def __init__(self, requests, H, g, T, dtype, L=1, E=None, seed=0, spare=3, strong=False, spread=1.0, gathered=False):
        gn = gen(seed + 1000 * H + T)
        self.ctx, self.new = [c for c, _ in requests], [m for _, m in requests]
        need = [max(0, -(-c // T)) for c in self.ctx]
        E = max(need + [1]) if E is None else E
        R, NB, N = len(requests), sum(need) + spare, sum(self.new)
        self.starts = [sum(self.new[:r]) for r in range(R + 1)]
        perm = torch.randperm(NB, generator=gn).to(torch.int32)
        self.tables, at = torch.full((L, R, E), -1, dtype=torch.int32), 0
        self.kc, self.vc = garbage((L, NB, T, H, 128), dtype, gn).to(DEV), garbage((L, NB, T, H, 128), dtype, gn).to(DEV)
        slots = []
        for r, n in enumerate(need):
            b = perm[at:at + n]
            at += n
            self.tables[:, r, :min(n, E)] = b[:E]
            pos = torch.arange(max(0, self.ctx[r]))
            slots.append(b[(pos // T)].long() * T + pos % T if n else pos)
        self.slots = torch.cat(slots).to(torch.int32)
        k = randn((L, self.slots.numel(), H, 128), gn)
        if strong:
            k[..., ::17] *= 8
        v = randn((L, self.slots.numel(), H, 128), gn) * spread
        self.rewrite(k.to(dtype), v.to(dtype))
        self.q = randn((L, N, H * g, 128), gn, dtype).to(DEV)
        self.scale, self.window, self.max_q = 128 ** -0.5, 0, max(self.new)
        self.many = self.max_q * g > 32      # probabilities rounded once
        self.gathered = torch.rand((L, R, E), generator=gn).to(DEV) * 50 if gathered else None

    def rewrite(self, k=None, v=None):
        self.k, self.v = self.k if k is None else k, self.v if v is None else v
        if self.slots.numel():
            rc.rc_kv_write(self.k.to(DEV), self.v.to(DEV), self.slots.to(DEV), self.kc, self.vc)

    def run(self, **kw):
        a = dict(dict(q=self.q, k=self.kc, v=self.vc, tables=self.tables.to(DEV), ctx_len=ints(self.ctx), q_start=ints(self.starts), max_q=self.max_q,
                      scale=self.scale, window=self.window, weights_in=self.gathered, want_weights=True), **kw)
        return rc.rc_kv_attend(**a)

    def check(self, r, tiny=2.0 ** -24):
        want, lse, weights, bound = ref.attend(self.q, self.kc, self.vc, self.tables, self.ctx, self.starts, self.scale, self.window, self.many, tiny,
                                               self.gathered)
        rows = [n for a, m in zip(self.starts, self.new) for n in range(a, a + m)]
        for got, x, b, name in ((r["out"][:, rows], want[:, rows], bound.out[:, rows], "out"), (r["lse"][:, rows], lse[:, rows], bound.lse[:, rows], "lse"),
                                (r["weights"], weights, bound.weights, "weights")):
            if got is None:
                continue
            got = got.cpu().double()
            # (which of the two a sum with an infinity in it becomes is left open)
            assert torch.equal(torch.isfinite(got), torch.isfinite(x)), name
            fine = torch.isfinite(x)
            off, b = (got - x).abs()[fine], b[fine]
            # (rows that see nothing are exact: no error, no bound)
            say(name, "largest error in bounds:", torch.where(b > 0, off / b, off).max().item() if off.numel() else 0.0)
            assert (off <= b).all(), name


WIDE = 40000        # entries of a table: items may be cut however short they are, and many rows go in tiles of 128 instead of 64

SHAPES = {
    "one token": [(1, 1)],
    "two": [(2, 1), (1, 1)],
    "a tile": [(16, 1), (17, 1), (15, 1)],
    "a run": [(32, 1), (33, 1), (31, 1), (64, 1)],
    "a step": [(128, 1), (129, 1), (127, 1), (256, 1), (257, 1)],
    "empty places": [(0, 1), (40, 1), (0, 1), (-3, 1), (70, 1), (0, 0), (5, 0)],
    "draft": [(100, 3), (3, 3), (64, 2), (131, 1)],
    "more queries than tokens": [(2, 3), (0, 3), (1, 2)],
    "cut": [(1300, 1), (20, 1), (3000, 1), (0, 1), (700, 1)],
    "prefill": [(50, 50), (90, 33), (0, 4), (130, 1), (64, 64)],
    "chunk": [(300, 90), (1500, 40), (90, 90)],
}


@pytest.mark.parametrize("H,g,T,dtype", [(2, 5, 16, HALF), (1, 1, 32, BF), (3, 4, 16, BF), (2, 8, 32, HALF), (1, 16, 16, BF), (2, 7, 32, HALF)])
@pytest.mark.parametrize("shape", sorted(SHAPES))
@pytest.mark.parametrize("E", [None, WIDE])
def test_attend(shape, H, g, T, dtype, E):
    say(shape, H, g, T, dtype, E)
    p = Problem(SHAPES[shape], H, g, T, dtype, E=E, strong=g == 5, gathered=H == 2)
    p.check(p.run())


@pytest.mark.parametrize("window", [1, 16, 33, 200, 100000])
@pytest.mark.parametrize("shape", ["draft", "cut", "chunk", "more queries than tokens"])
@pytest.mark.parametrize("T,dtype,E", [(16, BF, None), (32, HALF, WIDE)])
def test_window(shape, window, T, dtype, E):
    say(shape, window, T, dtype, E)
    p = Problem(SHAPES[shape], 2, 4, T, dtype, E=E, gathered=True)
    p.window = window
    p.check(p.run())


@pytest.mark.parametrize("T,g", [(16, 1), (32, 5), (16, 8)])
@pytest.mark.parametrize("q,E", [(1, None), (3, None), (20, None), (20, WIDE)])
def test_holes_layers_and_shared_blocks(T, g, q, E):
    say(T, g, q, E)
    p = Problem([(200, q), (1250, q), (333, q), (900, q)], 2, g, T, HALF, L=3, E=E, seed=q, gathered=True)
    t = p.tables
    t[0, 0, :] = -1                                  # a request whose table is empty
    t[1, 1, ::3], t[1, 2, 0], t[1, 2, 1] = -7, 1 << 30, p.kc.shape[1]
    t[2, 2, :3] = t[2, 0, :3]                        # blocks that two requests share, and one twice
    t[2, 1, 4] = t[2, 1, 5]
    t[0, 3, 2:20] = -1                               # runs of nothing
    t[1, 3, 1:25] = -1
    t[2, 3, 20:] = -1                                # ... the step's own tokens among them
    p.check(p.run())


def test_table_shorter_than_the_context():
    for q, g in ((1, 5), (30, 4)):
        p = Problem([(400, q), (100, q)], 2, g, 16, BF, E=13)
        p.check(p.run())


@pytest.mark.parametrize("m,g,T,dtype", [(1, 4, 16, HALF), (1, 1, 32, BF), (4, 7, 32, HALF), (6, 5, 16, BF), (40, 2, 16, BF)])
def test_tables_with_room_for_more_than_the_caches_hold(m, g, T, dtype):
    """Rows of a table that could list more blocks than a last-level cache holds and list some: the calls that load tokens without keeping them."""
    p = Problem([(700, m), (3000, m), (33, m), (0, m)], 2, g, T, dtype, E=500_000 // T)
    p.check(p.run())


@pytest.mark.parametrize("dtype", [HALF, BF])
@pytest.mark.parametrize("m,g,E", [(1, 4, None), (5, 3, None), (4, 8, None), (40, 2, None), (40, 2, WIDE), (15, 4, None)])
def test_infinities_and_nans_reach_only_the_rows_that_see_them(m, g, dtype, E):
    say(m, g, dtype, E)
    n = 300
    p = Problem([(n, m), (n, m), (n, m)], 2, g, 16, dtype, E=E)
    k, v = p.k.clone(), p.v.clone()
    v[0, n - 1, 0, 70] = math.nan                    # the last token: seen by the last query token only
    v[0, n - 1, 0, 71], v[0, n - 1, 0, 127] = math.inf, -math.inf
    v[0, n + 40, 1, 0] = math.nan                    # seen by all
    v[0, 2 * n + 299, 1, 5], v[0, 2 * n + 298, 1, 5] = math.inf, -math.inf
    if m > 1:
        k[0, n - 2, 1, 3] = math.inf                 # ... and a key of head 1
    p.rewrite(k, v)
    r = p.run()
    p.check(r)
    assert not torch.isfinite(r["out"]).all() and torch.isfinite(r["out"]).any()


def test_rows_that_do_not_see_a_nan_keep_their_bits():
    for m, g, E in ((3, 4, None), (7, 4, None), (40, 2, None), (40, 2, WIDE)):
        p = Problem([(300, m)], 2, g, 16, HALF, E=E)
        clean = p.run(want_weights=False)
        v = p.v.clone()
        v[0, 299] = math.nan
        p.rewrite(v=v)
        r = p.run(want_weights=False)
        assert torch.equal(r["out"][0, :m - 1], clean["out"][0, :m - 1]) and torch.equal(r["lse"], clean["lse"]) and r["out"][0, m - 1].isnan().all()


def test_queries_that_are_not_finite_stay_in_their_rows():
    p = Problem([(500, 1), (60, 1)], 2, 4, 16, HALF)
    clean = p.run()
    p.q[0, 0, 1, 5], p.q[0, 1, 7, 9] = math.nan, math.inf
    r = p.run()
    hit = torch.zeros((1, 2, 8), dtype=torch.bool, device=DEV)
    hit[0, 0, 1] = hit[0, 1, 7] = True
    assert torch.equal(r["out"][~hit], clean["out"][~hit]) and torch.equal(r["lse"][~hit], clean["lse"][~hit])
    assert r["out"][0, 0, 1].isnan().all() and r["out"][0, 1, 7].isnan().all()


@pytest.mark.parametrize("dtype", [HALF, BF])
@pytest.mark.parametrize("m,g", [(2, 3), (8, 4), (16, 1), (30, 1), (40, 2), (300, 3)])
@pytest.mark.parametrize("window", [0, 1, 20, 150])
def test_rows_that_are_not_finite_weigh_on_what_they_see_alone(m, g, window, dtype):
    say(m, g, window, dtype)
    p = Problem([(300, m), (320, m), (310, m)], 2, g, 16, dtype)
    p.window = window
    p.q[0, m // 3, 1 % g, 5] = math.nan
    # a key of the third request that makes a score of infinity for the rows that see it, from the middle of the step on
    p.q[..., 3] = p.q[..., 3].abs() + 0.25
    p.k[0, 300 + 320 + 310 - 1 - m // 2, 1, 3] = math.inf
    p.rewrite()
    r = p.run()
    p.check(r)
    assert not torch.isfinite(r["weights"]).all() and (window == 0 or torch.isfinite(r["weights"]).any())


@pytest.mark.parametrize("dtype,spread", [(HALF, 2.0 ** -17), (HALF, 3000.0), (BF, 1e-30), (BF, 1e30), (BF, 2.0 ** -118)])
@pytest.mark.parametrize("m", [1, 30])
def test_values_of_any_size(dtype, spread, m):
    p = Problem([(200, m), (77, m)], 2, 4, 16, dtype, spread=spread)
    # beside the relative bound only the smallest number of the type
    p.check(p.run(), tiny=2.0 ** -25 if dtype == HALF else 2.0 ** -133)


@pytest.mark.parametrize("scale", [1e-4, 0.5, 4.0])
@pytest.mark.parametrize("m", [1, 30])
def test_sharp_and_flat_softmax(scale, m):
    """Scores up to several hundreds: the reference is moved again and again."""
    p = Problem([(900, m), (1100, m)], 1, 5, 16, HALF, E=None if scale < 1 else WIDE, strong=True)
    p.scale = scale
    p.check(p.run())


@pytest.mark.parametrize("dtype", [HALF, BF])
@pytest.mark.parametrize("g,n,E", [(1, 40, None), (4, 64, None), (16, 128, WIDE), (17, 97, None), (25, 110, WIDE), (32, 128, None)])
@pytest.mark.parametrize("weigh", [False, True])
def test_few_rows_lose_nothing_of_their_probabilities(g, n, E, dtype, weigh):
    """With up to 32 rows a probability is the sum of two 16-bit numbers: outputs that nearly cancel are as close as that makes them."""
    say(g, n, E, dtype, weigh)
    p = Problem([(n, 1)], 1, g, 16, dtype, E=E)
    q, k, v = cache_cancelling.problem(g, n, dtype, gen(g))
    p.rewrite(torch.nn.functional.pad(k[None, :, None, None], (0, 127)), v[None, :, None])
    p.q = torch.nn.functional.pad(q[None, None, :, None], (0, 127)).to(DEV)
    p.scale = 1.0
    weights = cache_cancelling.weights(q, k)
    off = (p.run(want_weights=weigh)["out"][0, 0].cpu().double() - weights @ v.double()).abs() / cache_cancelling.bound(weights, v.double(), dtype)
    say("largest error in bounds:", off.max().item())
    assert off.max() <= 1


def test_scores_that_climb():
    for m, g, E in ((1, 4, None), (6, 4, None), (20, 4, None), (20, 4, 20 * WIDE)):
        n, H = 640, 1
        p = Problem([(n, m)], H, g, 16, BF, E=E)
        k = torch.zeros((1, n, H, 128))
        k[0, :, 0, 0] = torch.arange(n) / 16.0
        p.rewrite(k.to(BF))
        p.q[..., 0] = 6.0
        p.scale = 1.0
        p.check(p.run())


def test_one_token_each_without_q_start_and_strided_queries():
    p = Problem([(100, 1), (40, 1), (0, 1)], 2, 3, 16, HALF)
    wide = torch.zeros((1, 3, 16, 128), dtype=HALF, device=DEV)
    wide[:, :, 5:11] = p.q
    a, b = p.run(), p.run(q=wide[:, :, 5:11], q_start=None)
    p.check(a)
    assert all(torch.equal(a[x], b[x]) for x in a)


def test_query_tokens_of_no_request_stay():
    p = Problem([(100, 2), (40, 3)], 2, 2, 16, BF)
    wide = torch.cat([p.q[:, :1], p.q, p.q[:, :2]], 1).contiguous()
    out, lse = torch.full_like(wide, 7.0), torch.full(wide.shape[:3], 7.0, device=DEV)
    r = p.run(q=wide, q_start=torch.tensor([1, 3, 6], dtype=torch.int32, device=DEV), out=out, lse=lse)
    want = p.run()
    assert torch.equal(r["out"][:, 1:6], want["out"]) and torch.equal(r["lse"][:, 1:6], want["lse"]) and torch.equal(r["weights"], want["weights"])
    for t in (out, lse):
        assert (t[:, 0] == 7).all() and (t[:, 6:] == 7).all()


def test_further_tokens_than_max_q_are_not_computed():
    for m, g in ((4, 2), (40, 2)):
        p = Problem([(100, m), (90, 2)], 2, g, 16, BF)
        out = torch.full_like(p.q, 7.0)
        full, r = p.run(), p.run(max_q=m // 2, out=out)
        assert torch.equal(r["out"][:, m // 2:m], torch.full_like(out[:, m // 2:m], 7.0))
        # which are a request's computed ones is told by their places: the last token stands at the context's end
        assert ((r["lse"] - full["lse"])[:, :m // 2].abs() <= 2.0 ** -11).all()


def test_wild_lengths_stay_in_bounds():
    """Starts that descend or lie outside, lengths beyond max_q, contexts beyond every table: nothing is read or written out of range."""
    p = Problem([(100, 2), (40, 3), (64, 1)], 2, 2, 16, BF)
    for starts in ([5, 2, 9, 1], [-4, 3, 100, 6], [0, 6, 6, 6], [2147483647, -2147483648, 0, 6]):
        for ctx in ([2147483647, -2147483648, 5], [100, 40, 64]):
            for max_q in (1, 3, 6, 1000):
                guard = torch.full((8, 4, 128), 7.0, dtype=BF, device=DEV)
                weights = torch.full((5, *p.tables.shape[1:]), 7.0, device=DEV)
                r = p.run(q_start=ints(starts), ctx_len=ints(ctx), max_q=max_q, out=guard[1:7].unsqueeze(0), weights_out=weights[2:3])
                torch.cuda.synchronize()
                assert (guard[0] == 7).all() and (guard[7] == 7).all() and r["lse"].shape == (1, 6, 4)
                assert (weights[:2] == 7).all() and (weights[3:] == 7).all()


def test_blocks_beyond_four_gigabytes():
    H, T = 16, 32
    n = (1 << 32) // (T * H * 128 * 2) + 40
    if torch.cuda.mem_get_info()[0] < 20 << 30:
        pytest.fail("too little free memory")
    kc, vc = (torch.zeros((1, n, T, H, 128), dtype=BF, device=DEV) for _ in range(2))
    g = gen(11)
    ids = torch.tensor([n - 1, 3, n - 7, n - 2], dtype=torch.int32)
    k, v = randn((1, 4 * T, H, 128), g, BF), randn((1, 4 * T, H, 128), g, BF)
    slots = (ids[:, None] * T + torch.arange(T, dtype=torch.int32)).reshape(-1)
    rc.rc_kv_write(k.to(DEV), v.to(DEV), slots.to(DEV), kc, vc)
    small = [torch.zeros((1, 4, T, H, 128), dtype=BF, device=DEV) for _ in range(2)]
    rc.rc_kv_write(k.to(DEV), v.to(DEV), torch.arange(4 * T, dtype=torch.int32, device=DEV), *small)
    assert torch.equal(kc[:, ids.long().to(DEV)], small[0]) and torch.equal(vc[:, ids.long().to(DEV)], small[1])
    for m in (1, 9):
        q, ctx, starts = randn((1, m, 32, 128), g, BF).to(DEV), ints([4 * T - 3]), ints([0, m])
        x = rc.rc_kv_attend(q, kc, vc, ids.reshape(1, 1, 4).to(DEV), ctx, starts, want_weights=True)
        y = rc.rc_kv_attend(q, *small, torch.arange(4, dtype=torch.int32, device=DEV).reshape(1, 1, 4), ctx, starts, want_weights=True)
        assert all(torch.equal(x[i], y[i]) for i in x)


@pytest.mark.parametrize("dtype", [HALF, BF])
def test_blocks_of_none(dtype):
    """Nothing is stored, nothing is seen, nothing is gathered."""
    none = torch.zeros((2, 0, 32, 3, 128), dtype=dtype, device=DEV)
    q, tables = torch.ones((2, 2, 6, 128), dtype=dtype, device=DEV), torch.zeros((2, 2, 50), dtype=torch.int32, device=DEV)
    before = torch.rand((2, 2, 50), device=DEV)
    r = rc.rc_kv_attend(q, none, none, tables, ints([40, 3]), weights_in=before)
    assert not r["out"].any() and (r["lse"] == -math.inf).all() and torch.equal(r["weights"], before)
    # no query token, no entry
    some = torch.zeros((2, 4, 32, 3, 128), dtype=dtype, device=DEV)
    assert torch.equal(rc.rc_kv_attend(q[:, :0], some, some, tables, ints([40, 3]), ints([0, 0, 0]), weights_in=before)["weights"], before)
    assert not rc.rc_kv_attend(q[:, :0], some, some, tables, ints([40, 3]), ints([0, 0, 0]), want_weights=True)["weights"].any()
    r = rc.rc_kv_attend(q, some, some, tables[:, :, :0].contiguous(), ints([40, 3]), want_weights=True)
    assert not r["out"].any() and (r["lse"] == -math.inf).all() and r["weights"].numel() == 0


# query tokens, query heads of a KV head, entries of a table: tiles of 16, 32, 64, 128 and 192 rows, items that are cut and whole ones
KERNELS = [(1, 4, None), (1, 4, WIDE), (5, 4, None), (5, 4, WIDE), (12, 4, None), (12, 4, WIDE), (40, 4, 5000), (40, 4, 20 * WIDE)]


@pytest.mark.parametrize("m,g,E", KERNELS + [(20, 5, 20 * WIDE), (1, 5, None), (1, 3, WIDE), (7, 7, None)])
@pytest.mark.parametrize("dtype", [HALF, BF])
def test_unwritten_memory_leaves_no_trace(m, g, E, dtype):
    """Places behind the contexts, in blocks that the tables list, and the workspace hold one thing or another: the results are the same bits."""
    say(m, g, E, dtype)
    p = Problem([(m + 37 * i, m) for i in range(24)], 2, g, 16, dtype, E=E)
    results = []
    need = rc.rc_kv_attend_workspace_size(p.kc, 24, p.tables.shape[2], 2 * g, p.q.shape[1], m, True)
    assert need > 0
    room = torch.empty(need, dtype=torch.uint8, device=DEV)
    for seed in (1, 2, 3):
        for pool in (p.kc, p.vc):
            pool.copy_(garbage(pool.shape, dtype, gen(seed)))
        p.rewrite()
        room.fill_((0, 0xff, 0x7f)[seed - 1])
        results.append(p.run(workspace=room))
    for r in results[1:]:
        assert all(torch.equal(r[x], results[0][x]) for x in r)
    assert torch.isfinite(results[0]["weights"]).all()


@pytest.mark.parametrize("m,g,E", KERNELS)
@pytest.mark.parametrize("n,keys", [(1, "any"), (40, "any"), (700, "climbing"), (6000, "equal"), (70000, "equal")])
def test_largest_bf16_values(n, keys, m, g, E):
    """All tokens have the same values, up to the largest of the type: so has every weighted mean of them."""
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
    p.rewrite(k.to(BF), v.expand(p.v.shape).to(BF))
    r = p.run()
    want = v.double().expand(r["out"].shape)
    # one rounding of the result, one of the probabilities where they are rounded once, sums and exponentials as in kv_reference.Bound
    h = torch.finfo(BF).eps / 2
    off = (r["out"].cpu().double() - want).abs()
    assert (off <= want.abs() * (h + (h if p.many else h * h) + 2.0 ** -11)).all(), off.max()
    # all probabilities of a row together are one
    assert torch.isfinite(r["lse"]).all() and ((r["weights"].double().sum(-1) - m * g).abs() <= m * g * 2.0 ** -11).all()


@pytest.mark.parametrize("m,g,E", KERNELS)
@pytest.mark.parametrize("first", [0, 37, 300, 650])
def test_some_large_bf16_values(m, g, E, first):
    """Large values from some token on beside ordinary and small ones."""
    say(m, g, E, first)
    p = Problem([(700, m), (90, m)], 2, g, 16, BF, E=E, seed=first)
    gn = gen(first)
    v = p.v.float()
    large = torch.rand(v.shape[:3], generator=gn) < 0.1
    large[:, :first] = False
    v[..., 32:64] *= torch.where(large, 2.0 ** 124, 1.0)[..., None]
    v[..., 64:96] *= 2.0 ** -60
    p.rewrite(v=v.to(BF))
    p.check(p.run(), tiny=2.0 ** -133)


@pytest.mark.parametrize("m,g,E", KERNELS)
@pytest.mark.parametrize("dtype", [HALF, BF])
@pytest.mark.parametrize("scale", [1e6, 1e8, 1e9, 1e10])
def test_huge_scores_give_means(m, g, E, dtype, scale):
    """However coarse scores are, an output lies between the least and the largest of its values, and a row's probabilities are one together."""
    say(m, g, E, dtype, scale)
    p = Problem([(300, m), (40, m)], 2, g, 16, dtype, E=E, strong=True)
    p.scale = scale
    r = p.run()
    out = r["out"].cpu().double()
    h = torch.finfo(dtype).eps / 2
    for i, n in enumerate(p.ctx):
        v = p.v[0, sum(p.ctx[:i]):][:n].double()
        for head in range(2 * g):
            got, x = out[0, p.starts[i]:p.starts[i + 1], head], v[:, head // g]
            room = 2 * (h + 2.0 ** -12) * x.abs().amax(0)
            assert (got >= x.amin(0) - room).all() and (got <= x.amax(0) + room).all()
    assert ((r["weights"].double().sum(-1) - 2 * m * g).abs() <= 2 * m * g * 2.0 ** -11).all()


@pytest.mark.parametrize("R", [65, 200, 1000])
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
    p = Problem([(max(c, 0), n) for c, n in zip(ctx, new)], 2, g, 16, HALF, E=E, gathered=True)
    p.check(p.run())


@pytest.mark.parametrize("T,E", [(16, 3), (32, 2), (16, 67)])
@pytest.mark.parametrize("m,g", [(1, 4), (5, 4), (12, 4), (40, 4)])
def test_window_behind_a_short_table(T, E, m, g):
    """Queries whose window has slid past what the table lists see nothing, whatever its last block holds."""
    for past in (8, 9, 15, 16, 17, 40):
        p = Problem([(E * T + past + m - 1, m), (max(m, E * T - 3), m)], 1, g, T, BF, E=E)
        p.window = 8
        last = p.tables[0, 0, E - 1].item()
        p.vc[0, last], p.kc[0, last] = math.nan, math.nan
        r = p.run()
        assert (r["out"][0, :m] == 0).all() and (r["lse"][0, :m] == -math.inf).all() and (r["weights"][0, 0] == 0).all(), past
        p.check(r)


@pytest.mark.parametrize("m", [1, 40])
@pytest.mark.parametrize("T,R,E", [(16, 1, (1 << 27) - 5), (32, 1, (1 << 26) - 3), (16, 1 << 10, 1 << 19)])
def test_largest_tables(T, R, E, m):
    """The longest tables there are (positions to 2^31 - 64), and 2^29 entries that are weighed: as in a table of the last entries alone, which are all that a window sees."""
    say(T, R, E, m)
    gn = gen(R)
    few = [(int(torch.randint(180, 300, (1,), generator=gn)), int(torch.randint(0, 2, (1,), generator=gn))) for _ in range(R - 1)]
    p = Problem([(20 * T, m)] + few, 1, 1, T, HALF, E=20)
    p.window = 100
    # only requests of one can be as long: many stand at the beginning of their tables
    at = E - 20 if R == 1 else 0
    tables = torch.full((1, R, E), -1, dtype=torch.int32, device=DEV)
    tables[:, :, at:at + 20] = p.tables.to(DEV)
    # (what this call needs: the size for up to 40 query tokens holds for 32 rows of the other kernels as well)
    r = p.run(tables=tables, ctx_len=ints([n + at * T for n in p.ctx]), workspace=torch.empty(5 << 30, dtype=torch.uint8, device=DEV))
    w = r["weights"]
    r["weights"] = w[:, :, at:at + 20].clone()
    w[:, :, at:at + 20] = 0
    assert not w.any()
    p.check(r)


# ---- streams, graphs, workspaces

@pytest.mark.parametrize("m,g", [(1, 5), (3, 8), (15, 4), (40, 3)])
@pytest.mark.parametrize("weigh", [False, True])
def test_same_bits_on_every_run_and_guard_behind_the_workspace(m, g, weigh):
    p = Problem([(2500, m), (40, m), (1200, m)], 2, g, 16, HALF, E=400)
    need = rc.rc_kv_attend_workspace_size(p.kc, 3, 400, 2 * g, 3 * m, m, weigh)
    assert need > 0
    room = torch.full((need + 4096,), 0xa5, dtype=torch.uint8, device=DEV)
    first = p.run(workspace=room[:need], want_weights=weigh)
    if weigh:
        p.check(first)
    for _ in range(4):
        room[:need].random_(0, 256)
        r = p.run(workspace=room[:need], want_weights=weigh)
        assert all(first[x] is None or torch.equal(r[x], first[x]) for x in r)
    assert (room[need:] == 0xa5).all()


def test_out_and_lse_are_the_same_bits_with_weights_and_without():
    for m, g in ((1, 5), (3, 8), (15, 4), (40, 3)):
        p = Problem([(2500, m), (40, m), (1200, m)], 2, g, 16, HALF, E=400)
        a, b, c = p.run(), p.run(want_weights=False), p.run(want_weights=False, want_lse=False)
        assert torch.equal(a["out"], b["out"]) and torch.equal(a["lse"], b["lse"]) and torch.equal(a["out"], c["out"]) and c["lse"] is None


# ---- evict

def evict_problem(L, R, E, T, seed, shared=0.3, holes=0.1, NB=None):
    g = gen(seed)
    NB = R * E + 7 if NB is None else NB
    ctx = torch.randint(0, E * T + 20, (R,), generator=g).tolist()
    ctx[0] = E * T - T // 2
    tables = torch.stack([torch.randperm(NB, generator=g)[:R * E].reshape(R, E) if NB >= R * E else torch.randint(0, NB, (R, E), generator=g)
                          for _ in range(L)]).to(torch.int32)
    if R > 1:
        n = int(E * shared)
        tables[:, 1:, :n] = tables[:, :1, :n]
    gone = torch.rand(tables.shape, generator=g) < holes
    tables[gone] = torch.randint(-3, 0, tables.shape, generator=g).to(torch.int32)[gone]
    tables[torch.rand(tables.shape, generator=g) < holes / 3] = NB + 5
    weights = torch.rand(tables.shape, generator=g) ** 6 * 100
    weights[torch.rand(tables.shape, generator=g) < 0.3] = 0.0
    keep = torch.randint(-1, E + 2, (R,), generator=g).tolist()
    keep[0] = E // 2
    refcount = torch.randint(1, 100, (L, NB), generator=g, dtype=torch.int32)
    return tables, weights, ctx, keep, refcount


def run_evict(tables, weights, ctx, keep, refcount, T, **kw):
    return rc.rc_kv_evict(tables.to(DEV), weights.to(DEV), ints(ctx), ints(keep), refcount.to(DEV), T, **kw)


def check_evict(r, want):
    for got, x in zip((r["tables"], r["refcount"], r["n_evicted"]), want):
        assert torch.equal(got.cpu(), x)


@pytest.mark.parametrize("L,R,E,T", [(1, 1, 1, 16), (1, 1, 2, 32), (2, 3, 7, 16), (1, 5, 63, 16), (3, 2, 64, 32), (2, 7, 65, 16), (1, 3, 300, 32),
                                     (2, 2, 1023, 16), (1, 2, 1024, 16), (1, 2, 1025, 16), (2, 1, 5000, 32), (1, 1, 16384, 16), (1, 2, 16385, 16),
                                     (1, 1, 40001, 32)])
@pytest.mark.parametrize("first,last", [(0, 1), (1, 2), (4, 1 << 40)])
def test_evict(L, R, E, T, first, last):
    say(L, R, E, T, first, last)
    tables, weights, ctx, keep, refcount = evict_problem(L, R, E, T, E + first)
    want = ref.evict(tables, weights, ctx, keep, refcount, T, first, last)
    check_evict(run_evict(tables, weights, ctx, keep, refcount, T, n_first=first, n_last=last), want)
    # in place, and with outputs of the caller's
    check_evict(run_evict(tables, weights, ctx, keep, refcount, T, n_first=first, n_last=last, in_place=True), want)
    out = dict(tables=torch.full(tables.shape, 77, dtype=torch.int32, device=DEV), refcount=torch.full(refcount.shape, 77, dtype=torch.int32, device=DEV),
               n_evicted=torch.full((L, R), 77, dtype=torch.int32, device=DEV))
    check_evict(run_evict(tables, weights, ctx, keep, refcount, T, n_first=first, n_last=last, out=out), want)


@pytest.mark.parametrize("E", [50, 700, 3000, 20000])
@pytest.mark.parametrize("kind", ["equal", "signs", "strange", "near", "few levels"])
def test_evict_weights_of_all_kinds(E, kind):
    say(E, kind)
    tables, weights, ctx, keep, refcount = evict_problem(1, 2, E, 16, E)
    g = gen(E + 1)
    if kind == "equal":
        weights.fill_(0.25)
    elif kind == "signs":
        weights = torch.where(torch.rand(weights.shape, generator=g) < 0.5, 0.0, -0.0) + torch.randint(-1, 2, weights.shape, generator=g) * 1e-40
    elif kind == "strange":
        pick = torch.tensor([math.nan, -math.nan, math.inf, -math.inf, 3e38, -3e38, 1e-45, 0.0, -0.0])
        weights = pick[torch.randint(0, 9, weights.shape, generator=g)]
    elif kind == "near":
        weights = torch.randint(0x3f800000, 0x3f800000 + E // 3, weights.shape, generator=g, dtype=torch.int32).view(torch.float32)
    else:
        weights = torch.randint(0, 3, weights.shape, generator=g).float()
    ctx[1] = E * 16
    for k in (0, 1, E // 3, E - 3, E):
        keep = [k, k]
        check_evict(run_evict(tables, weights, ctx, keep, refcount, 16), ref.evict(tables, weights, ctx, keep, refcount, 16, 1, 1))


def test_evict_blocks_that_many_requests_hold():
    """Every request holds the same few blocks, some twice: a reference for each entry that left."""
    tables, weights, ctx, keep, refcount = evict_problem(2, 50, 40, 16, 3, holes=0.0, NB=9)
    refcount.fill_(1000)
    keep = [10] * 50
    check_evict(run_evict(tables, weights, ctx, keep, refcount, 16), ref.evict(tables, weights, ctx, keep, refcount, 16, 1, 1))


def test_evict_from_four_million_tables():
    R, E, T = (1 << 22) + 5, 1025, 16
    g = gen(8)
    ids, weights = torch.randint(0, 4000, (3, E), generator=g, dtype=torch.int32), torch.rand((3, E), generator=g)
    which = torch.arange(R, device=DEV) % 3
    tables, refcount = ids.to(DEV)[which][None], torch.full((1, 4000), 1 << 30, dtype=torch.int32)
    ctx, keep = torch.full((R,), E * T, dtype=torch.int32, device=DEV), torch.full((R,), E - 1, dtype=torch.int32, device=DEV)
    got = rc.rc_kv_evict(tables, weights.to(DEV)[which][None], ctx, keep, refcount.to(DEV), T, in_place=True)
    want = ref.evict(ids[None], weights[None], [E * T] * 3, [E - 1] * 3, refcount, T, 1, 1)[0]
    assert (got["n_evicted"] == 1).all()
    for i in range(3):
        assert (got["tables"][0, i::3] == want[0, i].to(DEV)).all()
        refcount[0, ids[i][want[0, i] < 0].item()] -= len(range(i, R, 3))
    assert torch.equal(got["refcount"].cpu(), refcount)


def test_evict_nothing():
    empty = torch.zeros((2, 0, 5), dtype=torch.int32)
    r = run_evict(empty, empty.float(), [], [], torch.tensor([[1, 2], [3, 4]], dtype=torch.int32), 16)
    assert r["refcount"].tolist() == [[1, 2], [3, 4]] and r["n_evicted"].shape == (2, 0)
    empty = torch.zeros((1, 2, 0), dtype=torch.int32)
    r = run_evict(empty, empty.float(), [5, 9], [0, 0], torch.zeros((1, 0), dtype=torch.int32), 32)
    assert r["n_evicted"].tolist() == [[0, 0]]


# ---- together

def test_steps_of_a_cache_that_evicts():
    """Store, attend and weigh, evict, remap a block that two requests came to share, attend: captured once and replayed, against eager steps and the
    definition."""
    T, H, g, n = 16, 2, 4, 400
    p = Problem([(n, 1), (n, 1), (250, 1)], H, g, T, HALF, E=30, spare=8)
    tables = p.tables.clone()
    tables[0, 1, :3] = tables[0, 0, :3]              # a shared prefix
    NB = p.kc.shape[1]
    refcount = torch.zeros((1, NB), dtype=torch.int32)
    for i in tables[tables >= 0].tolist():
        refcount[0, i] += 1
    d = dict(tables=tables.to(DEV), refcount=refcount.to(DEV), weights=torch.zeros(tables.shape, device=DEV), ctx=ints(p.ctx), keep=ints([20, 12, 100]),
             slots=ints([tables[0, r, (c - 1) // T].item() * T + (c - 1) % T for r, c in enumerate(p.ctx)]))
    k, v, q = (torch.zeros((1, 3, x, 128), dtype=HALF, device=DEV) for x in (H, H, H * g))
    out, lse, n_evicted = torch.empty_like(q), torch.empty((1, 3, H * g), device=DEV), torch.zeros((1, 3), dtype=torch.int32, device=DEV)
    room = torch.empty(rc.rc_kv_attend_workspace_size(p.kc, 3, 30, H * g, 3, 1, True), dtype=torch.uint8, device=DEV)

    def step():
        rc.rc_kv_write(k, v, d["slots"], p.kc, p.vc)
        rc.rc_kv_attend(q, p.kc, p.vc, d["tables"], d["ctx"], weights_in=d["weights"], weights_out=d["weights"], workspace=room, out=out, lse=lse)
        rc.rc_kv_evict(d["tables"], d["weights"], d["ctx"], d["keep"], d["refcount"], T, out=dict(tables=d["tables"], refcount=d["refcount"], n_evicted=n_evicted))

    inputs = [[randn(x.shape, gen(50 * i + j), HALF) for j, x in enumerate((k, v, q))] for i in range(5)]
    first = {x: t.clone() for x, t in d.items()}

    def load(i):
        for t, x in zip((k, v, q), inputs[i]):
            t.copy_(x)

    # eager, against the definition
    eager = []
    for i in range(5):
        load(i)
        before = {x: t.clone() for x, t in d.items()}
        step()
        torch.cuda.synchronize()
        want = ref.attend(q, p.kc, p.vc, before["tables"], p.ctx, p.starts, p.scale, 0, False, gathered=before["weights"])
        for got, x, b in zip((out, lse, d["weights"]), want[:3], (want[3].out, want[3].lse, want[3].weights)):
            assert ((got.cpu().double() - x).abs() <= b).all()
        left = ref.evict(before["tables"].cpu(), d["weights"].cpu(), p.ctx, d["keep"].tolist(), before["refcount"].cpu(), T, 1, 1)
        check_evict(dict(tables=d["tables"], refcount=d["refcount"], n_evicted=n_evicted), left)
        eager.append([t.clone() for t in (out, lse, d["tables"], d["refcount"], d["weights"])])
    assert (d["tables"] >= 0).sum(-1).tolist() == [[20, 12, 16]]
    # the second request's newest sealed block turns out to be the first one's: remapped, attended over
    e = 5
    while tables[0, 1, e].item() not in d["tables"][0, 1].tolist():
        e += 1
    kept = next(x for x in d["tables"][0, 0].tolist() if x >= 0)
    m = rc.rc_remap_block_table(d["tables"], tables[0, 1, e:e + 1].to(DEV), ints([kept]), ints([[0]]), 1, NB, d["refcount"])
    assert m["tables"][0, 1, e].item() == kept and m["n_remapped"].tolist() == [1]
    r = rc.rc_kv_attend(q, p.kc, p.vc, m["tables"], d["ctx"])
    want = ref.attend(q, p.kc, p.vc, m["tables"], p.ctx, p.starts, p.scale, 0, False)
    assert ((r["out"].cpu().double() - want[0]).abs() <= want[3].out).all()
    # captured, from the same beginning, on another stream than the eager steps, with eager work between the replays
    for x, t in first.items():
        d[x].copy_(t)
    load(0)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for x, t in first.items():
        d[x].copy_(t)
    for i in range(5):
        load(i)
        graph.replay()
        torch.cuda.synchronize()
        for got, x in zip((out, lse, d["tables"], d["refcount"], d["weights"]), eager[i]):
            assert torch.equal(got, x), i
        rc.rc_kv_attend(q, p.kc, p.vc, d["tables"], d["ctx"], weights_in=d["weights"])


def test_another_stream():
    p = Problem([(2500, 1), (40, 1), (1200, 1)], 2, 5, 16, HALF, E=400)
    want = p.run()
    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    args = dict(tables=p.tables.to(DEV), ctx_len=ints(p.ctx), q_start=ints(p.starts))
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):
        r = p.run(**args)
    torch.cuda.current_stream().wait_stream(other)
    assert all(torch.equal(r[x], want[x]) for x in r)


@pytest.mark.parametrize("g,m", [(33, 1), (64, 2), (200, 1), (1024, 1)])
def test_many_heads_of_a_kv_head(g, m):
    p = Problem([(300, m), (45, m), (0, m)], 1, g, 16, HALF, gathered=True)
    p.check(p.run())


@pytest.mark.parametrize("R,m,E", [(1, 700, 60), (3, 300, 60), (70, 40, 30), (130, 30, 30), (2, 900, 5000)])
def test_row_tiles_of_few_and_many_requests(R, m, E):
    """Lanes that count the tiles of one request together, or of one request each; stretches that begin in any tile."""
    gn = gen(R)
    requests = [(int(torch.randint(m, 480, (1,), generator=gn)) if E < 1000 and m < 480 else m + 60, int(torch.randint(1, m + 1, (1,), generator=gn))) for _ in range(R)]
    requests[R // 2] = (max(m, 470), m)
    p = Problem(requests, 2, 3, 16, BF, E=E, gathered=True)
    p.check(p.run())

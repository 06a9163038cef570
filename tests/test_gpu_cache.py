"""The 4-bit cache on the GPU: tokens quantised into it bit by bit as defined, blocks read back exactly, attention within the bound
that its arithmetic allows (tests/cache_reference.py).  Needs a real MI355X."""
import ctypes
import math
import sys

import pytest
import torch

from paper_2507_21433_amd import binding as rc
from tests import cache_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HALF, BF = torch.float16, torch.bfloat16


def say(*msg):
    print("[gpu-case]", *msg, flush=True)
    sys.stdout.flush()


def randn(shape, g, dtype=torch.float32):
    return torch.randn(shape, generator=g, dtype=torch.float32).to(dtype)


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def garbage(cache, g):
    """Any bytes, NaN exponents among them: what memory holds that was never written."""
    cache.copy_(torch.randint(0, 256, cache.shape, generator=g, dtype=torch.uint8))
    return cache


# ---- write and read

@pytest.mark.parametrize("dtype", [HALF, BF])
@pytest.mark.parametrize("lead", [0.0, 1.0, 7.0, 6.99, 2.0 ** -20, 65504.0, 3e38, 1e-38, math.inf, math.nan])
def test_every_pattern_is_quantised_as_defined(dtype, lead):
    say(dtype, lead)
    n = 4096
    x = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(dtype).reshape(n, 16)
    k = torch.zeros((1, n, 2, 128), dtype=dtype)
    # sixteen patterns beside a leading value, and the same patterns in groups that they rule themselves
    k[0, :, 0, :16], k[0, :, 0, 31], k[0, :, 1, 32:48], k[0, :, 1, 100:116] = x, lead, x, -x
    v = k.flip(3).contiguous()
    slots = torch.arange(n, dtype=torch.int32)
    cache = rc.cache_tensor(1, n // 16, 16, 2, DEV)
    rc.rc_cache_write(k.to(DEV), v.to(DEV), slots.to(DEV), cache)
    want = ref.write(torch.zeros(cache.shape, dtype=torch.uint8), k, v, slots)
    assert torch.equal(cache.cpu(), want)
    ids = torch.arange(n // 16, dtype=torch.int32)
    got, exact = rc.rc_cache_read(cache, ids.to(DEV), dtype), ref.read(want, ids)
    for a, b in zip(got, exact):
        assert torch.equal(torch.nan_to_num(a.cpu().double(), nan=1e300), torch.nan_to_num(b, nan=1e300))


@pytest.mark.parametrize("L,T,H,N,dtype", [(1, 16, 1, 1, HALF), (1, 16, 8, 3, BF), (3, 32, 5, 16, HALF), (2, 16, 16, 17, BF), (1, 32, 4, 33, BF),
                                           (2, 16, 10, 64, HALF), (1, 16, 3, 131, BF), (2, 32, 8, 96, HALF)])
@pytest.mark.parametrize("order", ["whole", "runs", "anywhere", "fused"])
def test_write(L, T, H, N, dtype, order):
    say(L, T, H, N, dtype, order)
    g = gen(N * 7 + H)
    NB = 2 * (N // T + 2)
    if order == "fused":
        wide = randn((L, N, 4 * H, 128), g, dtype).to(DEV)
        k, v = wide[:, :, 2 * H:3 * H], wide[:, :, 3 * H:]
    else:
        k, v = randn((L, N, H, 128), g, dtype).to(DEV), randn((L, N, H, 128), g, dtype).to(DEV)
    if order == "whole":
        slots = torch.arange(N, dtype=torch.int32) + T
    elif order == "runs":
        slots = torch.arange(N, dtype=torch.int32) + 5
        slots[N // 2:] += 7
    else:
        slots = torch.randperm(NB * T, generator=g)[:N].to(torch.int32)
    if N > 2:
        slots[N // 3], slots[N - 1] = -1, NB * T     # neither is stored
    cache = garbage(torch.zeros((L, NB, H, T // 16, 2176), dtype=torch.uint8), g)
    got = cache.to(DEV)
    rc.rc_cache_write(k, v, slots.to(DEV), got)
    assert torch.equal(got.cpu(), ref.write(cache, k.cpu(), v.cpu(), slots))


def test_write_leaves_other_layers_blocks_and_the_room_behind():
    g = gen(3)
    L, NB, T, H, N = 3, 6, 32, 3, 40
    room = garbage(torch.zeros((L, NB + 2, H, T // 16, 2176), dtype=torch.uint8), g)
    dev = room.to(DEV)
    k, v = randn((L, N, H, 128), g, HALF), randn((L, N, H, 128), g, HALF)
    slots = torch.arange(11, 11 + N, dtype=torch.int32)
    rc.rc_cache_write(k.to(DEV), v.to(DEV), slots.to(DEV), dev[:, 1:NB + 1])
    want = room.clone()
    want[:, 1:NB + 1] = ref.write(room[:, 1:NB + 1], k, v, slots)
    assert torch.equal(dev.cpu(), want)


@pytest.mark.parametrize("L,T,H,n,dtype", [(1, 16, 1, 1, HALF), (2, 32, 5, 7, BF), (3, 16, 16, 5, BF), (1, 32, 8, 33, HALF)])
def test_read(L, T, H, n, dtype):
    say(L, T, H, n, dtype)
    g = gen(n)
    NB = n + 3
    cache = garbage(torch.zeros((L, NB, H, T // 16, 2176), dtype=torch.uint8), g)
    # powers that the type holds, and NaNs
    low, high = ref.LIMITS[dtype]
    exponents = torch.randint(low + 127, high + 128, cache[..., 2048:].shape, generator=g)
    exponents[torch.rand(exponents.shape, generator=g) < 0.02] = 255
    cache[..., 2048:] = exponents.to(torch.uint8)
    ids = torch.randint(0, NB, (n,), generator=g, dtype=torch.int32)
    if n > 3:
        ids[1], ids[2] = -1, NB
    room = torch.full((L, n + 2, T, H, 128), 7.0, dtype=dtype, device=DEV), torch.full((L, n + 2, T, H, 128), 7.0, dtype=dtype, device=DEV)
    rc.rc_cache_read(cache.to(DEV), ids.to(DEV), k=room[0][:, 1:n + 1], v=room[1][:, 1:n + 1])
    for x, want in zip(room, ref.read(cache, ids)):
        # 6 * 2^high is beyond the largest code that a writer makes there, but a number of the type all the same
        assert torch.equal(torch.nan_to_num(x[:, 1:n + 1].cpu().double(), nan=1e300), torch.nan_to_num(want, nan=1e300))
        assert (x[:, 0] == 7).all() and (x[:, n + 1] == 7).all()


def test_nothing_to_do():
    cache = rc.cache_tensor(1, 4, 16, 2, DEV)
    k = torch.zeros((1, 0, 2, 128), dtype=HALF, device=DEV)
    rc.rc_cache_write(k, k, torch.zeros(0, dtype=torch.int32, device=DEV), cache)
    a, b = rc.rc_cache_read(cache, torch.zeros(0, dtype=torch.int32, device=DEV), HALF)
    assert a.numel() == b.numel() == 0 and not cache.any()


# ---- attend

class Problem:
    """Requests of (cached tokens, query tokens) over a cache whose written blocks lie anywhere among unwritten ones."""

    def __init__(self, requests, H, g, T, dtype, L=1, E=None, seed=0, spare=3, strong=False, spread=1.0):
        gn = gen(seed + 1000 * H + T)
        self.ctx, self.new = [c for c, _ in requests], [m for _, m in requests]
        need = [max(0, -(-c // T)) for c in self.ctx]
        E = max(need + [1]) if E is None else E
        R, NB, N = len(requests), sum(need) + spare, sum(self.new)
        self.starts = [sum(self.new[:r]) for r in range(R + 1)]
        perm = torch.randperm(NB, generator=gn).to(torch.int32)
        self.tables, at = torch.full((L, R, E), -1, dtype=torch.int32), 0
        self.cache = garbage(torch.zeros((L, NB, H, T // 16, 2176), dtype=torch.uint8), gn).to(DEV)
        slots = []
        for r, n in enumerate(need):
            b = perm[at:at + n]
            at += n
            self.tables[:, r, :min(n, E)] = b[:E]
            pos = torch.arange(max(0, self.ctx[r]))
            slots.append(b[(pos // T)].long() * T + pos % T if n else pos)
        slots = torch.cat(slots).to(torch.int32)
        k = randn((L, slots.numel(), H, 128), gn, torch.float32)
        if strong:
            k[..., ::17] *= 8
        v = randn((L, slots.numel(), H, 128), gn, torch.float32) * spread
        self.k, self.v, self.slots = k.to(dtype), v.to(dtype), slots
        if slots.numel():
            rc.rc_cache_write(self.k.to(DEV), self.v.to(DEV), slots.to(DEV), self.cache)
        self.q = randn((L, N, H * g, 128), gn, dtype).to(DEV)
        self.scale, self.window, self.max_q = 128 ** -0.5, 0, max(self.new)
        self.many = self.max_q * g > 16      # probabilities rounded once

    def run(self, **kw):
        i = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
        a = dict(dict(q=self.q, cache=self.cache, tables=self.tables.to(DEV), ctx_len=i(self.ctx), q_start=i(self.starts), max_q=self.max_q,
                      scale=self.scale, window=self.window), **kw)
        return rc.rc_cache_attend(**a)

    def check(self, r):
        want, lse, bound = ref.attend(self.q, self.cache, self.tables, self.ctx, self.starts, self.scale, self.window, self.many)
        rows = [n for a, m in zip(self.starts, self.new) for n in range(a, a + m)]
        for got, x, b, name in ((r["out"], want, bound.out, "out"), (r["lse"], lse, bound.lse, "lse")):
            got, x, b = got[:, rows].cpu().double(), x[:, rows], b[:, rows]
            assert torch.equal(got.isnan(), x.isnan()), name
            assert torch.equal(got == -math.inf, x == -math.inf) and torch.equal(got == math.inf, x == math.inf), name
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
    p = Problem(SHAPES[shape], H, g, T, dtype, E=E, strong=g == 5)
    p.check(p.run())


@pytest.mark.parametrize("window", [1, 16, 33, 200, 100000])
@pytest.mark.parametrize("shape", ["draft", "cut", "chunk", "more queries than tokens"])
@pytest.mark.parametrize("T,dtype,E", [(16, BF, None), (32, HALF, WIDE)])
def test_window(shape, window, T, dtype, E):
    say(shape, window, T, dtype, E)
    p = Problem(SHAPES[shape], 2, 4, T, dtype, E=E)
    p.window = window
    p.check(p.run())


@pytest.mark.parametrize("T,g", [(16, 1), (32, 5), (16, 8)])
@pytest.mark.parametrize("q,E", [(1, None), (3, None), (20, None), (20, WIDE)])
def test_holes_layers_and_shared_blocks(T, g, q, E):
    say(T, g, q, E)
    p = Problem([(200, q), (1250, q), (333, q)], 2, g, T, HALF, L=3, E=E, seed=q)
    t = p.tables
    t[0, 0, :] = -1                                  # a request whose table is empty
    t[1, 1, ::3], t[1, 2, 0], t[1, 2, 1] = -7, 1 << 30, p.cache.shape[1]
    t[2, 2, :3] = t[2, 0, :3]                        # blocks that two requests share, and one twice
    t[2, 1, 4] = t[2, 1, 5]
    p.check(p.run())


def test_table_shorter_than_the_context():
    for q, g in ((1, 5), (30, 4)):
        p = Problem([(400, q), (100, q)], 2, g, 16, BF, E=13)
        p.check(p.run())


@pytest.mark.parametrize("m,g,T,dtype", [(1, 4, 16, HALF), (1, 1, 32, BF), (4, 7, 32, HALF), (6, 5, 16, BF), (40, 2, 16, BF)])
def test_tables_with_room_for_more_than_the_caches_hold(m, g, T, dtype):
    """Rows of a table that could list 800 MB of cache and list some KB: the calls that load codes without keeping them."""
    E = 1_500_000 // T
    p = Problem([(700, m), (3000, m), (33, m), (0, m)], 2, g, T, dtype, E=E)
    p.check(p.run())


@pytest.mark.parametrize("dtype", [HALF, BF])
@pytest.mark.parametrize("m,g,E", [(1, 4, None), (5, 3, None), (4, 8, None), (40, 2, None), (40, 2, WIDE), (15, 4, None)])
def test_nan_reaches_only_the_rows_that_see_it(m, g, dtype, E):
    say(m, g, dtype, E)
    n = 300
    p = Problem([(n, m), (n, m)], 2, g, 16, dtype, E=E)
    slot = lambda r, pos: p.tables[0, r, pos // 16].item() * 16 + pos % 16
    k, v = p.k[:, :1].clone(), p.v[:, :1].clone()
    v[0, 0, 0, 70] = math.nan                        # head 0, group 2
    put = lambda k, v, s: rc.rc_cache_write(k.to(DEV), v.to(DEV), torch.tensor([s], dtype=torch.int32, device=DEV), p.cache)
    put(k, v, slot(0, n - 1))                        # the last token: seen by the last query token only
    put(k, v, slot(1, 40))                           # seen by all
    if m > 1:
        k[0, 0, 1, 3] = math.inf                     # ... and a key of head 1
        put(k, v, slot(0, n - 2))
    r = p.run()
    p.check(r)
    assert r["out"].isnan().any() and not r["out"].isnan().all()


def test_queries_that_are_not_finite_stay_in_their_rows():
    p = Problem([(500, 1), (60, 1)], 2, 4, 16, HALF)
    clean = p.run()
    p.q[0, 0, 1, 5], p.q[0, 1, 7, 9] = math.nan, math.inf
    r = p.run()
    hit = torch.zeros((1, 2, 8), dtype=torch.bool, device=DEV)
    hit[0, 0, 1] = hit[0, 1, 7] = True
    assert torch.equal(r["out"][~hit], clean["out"][~hit]) and torch.equal(r["lse"][~hit], clean["lse"][~hit])
    assert r["out"][0, 0, 1].isnan().all() and r["out"][0, 1, 7].isnan().all()


@pytest.mark.parametrize("dtype,spread", [(HALF, 2.0 ** -17), (HALF, 3000.0), (BF, 1e-30), (BF, 1e30)])
@pytest.mark.parametrize("m", [1, 30])
def test_values_of_any_size(dtype, spread, m):
    p = Problem([(200, m), (77, m)], 2, 4, 16, dtype, spread=spread)
    # beside the relative bound only the smallest number of the type
    want, lse, bound = ref.attend(p.q, p.cache, p.tables, p.ctx, p.starts, p.scale, 0, p.many, tiny=2.0 ** -25 if dtype == HALF else 2.0 ** -133)
    assert ((p.run()["out"].cpu().double() - want).abs() <= bound.out).all()


@pytest.mark.parametrize("scale", [1e-4, 0.5, 4.0])
@pytest.mark.parametrize("m", [1, 30])
def test_sharp_and_flat_softmax(scale, m):
    """Scores up to several hundreds: the reference is moved again and again."""
    p = Problem([(900, m), (1100, m)], 1, 5, 16, HALF, E=None if scale < 1 else WIDE, strong=True)
    # scores that climb along the context, so that every run of tokens passes the last one's reference
    p.scale = scale
    p.check(p.run())


def test_scores_that_climb():
    for m, g, E in ((1, 4, None), (6, 4, None), (20, 4, None), (20, 4, 20 * WIDE)):
        n, H = 640, 1
        p = Problem([(n, m)], H, g, 16, BF, E=E)
        k = torch.zeros((1, n, H, 128))
        k[0, :, 0, 0] = torch.arange(n) / 16.0
        rc.rc_cache_write(k.to(BF).to(DEV), p.v.to(DEV), p.slots.to(DEV), p.cache)
        p.q[..., 0] = 6.0
        p.scale = 1.0
        p.check(p.run())


def test_one_token_each_without_q_start_and_strided_queries():
    p = Problem([(100, 1), (40, 1), (0, 1)], 2, 3, 16, HALF)
    wide = torch.zeros((1, 3, 16, 128), dtype=HALF, device=DEV)
    wide[:, :, 5:11] = p.q
    a, b = p.run(), p.run(q=wide[:, :, 5:11], q_start=None)
    p.check(a)
    assert torch.equal(a["out"], b["out"]) and torch.equal(a["lse"], b["lse"])


def test_query_tokens_of_no_request_stay():
    p = Problem([(100, 2), (40, 3)], 2, 2, 16, BF)
    wide = torch.cat([p.q[:, :1], p.q, p.q[:, :2]], 1).contiguous()
    out, lse = torch.full_like(wide, 7.0), torch.full(wide.shape[:3], 7.0, device=DEV)
    r = p.run(q=wide, q_start=torch.tensor([1, 3, 6], dtype=torch.int32, device=DEV), out=out, lse=lse)
    want = p.run()
    assert torch.equal(r["out"][:, 1:6], want["out"]) and torch.equal(r["lse"][:, 1:6], want["lse"])
    for t in (out, lse):
        assert (t[:, 0] == 7).all() and (t[:, 6:] == 7).all()


def test_wild_lengths_stay_in_bounds():
    """Starts that descend or lie outside, lengths beyond max_q, contexts beyond every table: nothing is read or written out of range."""
    p = Problem([(100, 2), (40, 3), (64, 1)], 2, 2, 16, BF)
    i = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    for starts in ([5, 2, 9, 1], [-4, 3, 100, 6], [0, 6, 6, 6], [2147483647, -2147483648, 0, 6]):
        for ctx in ([2147483647, -2147483648, 5], [100, 40, 64]):
            for max_q in (1, 3, 6, 1000):
                guard = torch.full((8, 4, 128), 7.0, dtype=BF, device=DEV)
                r = p.run(q_start=i(starts), ctx_len=i(ctx), max_q=max_q, out=guard[1:7].unsqueeze(0))
                torch.cuda.synchronize()
                assert (guard[0] == 7).all() and (guard[7] == 7).all() and r["lse"].shape == (1, 6, 4)


def test_blocks_beyond_four_gigabytes():
    H, T = 16, 32
    n = (1 << 32) // (H * 2 * 2176) + 40
    if torch.cuda.mem_get_info()[0] < 12 << 30:
        pytest.fail("too little free memory")
    cache = torch.zeros((1, n, H, 2, 2176), dtype=torch.uint8, device=DEV)
    g = gen(11)
    ids = torch.tensor([n - 1, 3, n - 7, n - 2], dtype=torch.int32)
    k, v = randn((1, 4 * T, H, 128), g, BF), randn((1, 4 * T, H, 128), g, BF)
    slots = (ids[:, None] * T + torch.arange(T, dtype=torch.int32)).reshape(-1)
    rc.rc_cache_write(k.to(DEV), v.to(DEV), slots.to(DEV), cache)
    small = rc.cache_tensor(1, 4, T, H, DEV)
    rc.rc_cache_write(k.to(DEV), v.to(DEV), torch.arange(4 * T, dtype=torch.int32, device=DEV), small)
    assert torch.equal(cache[:, ids.long().to(DEV)], small)
    a, b = rc.rc_cache_read(cache, ids.to(DEV), BF), rc.rc_cache_read(small, torch.arange(4, dtype=torch.int32, device=DEV), BF)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    q, ctx = randn((1, 1, 32, 128), g, BF).to(DEV), torch.tensor([4 * T - 3], dtype=torch.int32, device=DEV)
    x = rc.rc_cache_attend(q, cache, ids.reshape(1, 1, 4).to(DEV), ctx)
    y = rc.rc_cache_attend(q, small, torch.arange(4, dtype=torch.int32, device=DEV).reshape(1, 1, 4), ctx)
    assert torch.equal(x["out"], y["out"]) and torch.equal(x["lse"], y["lse"])


# ---- streams, graphs, workspaces

@pytest.mark.parametrize("m,g", [(1, 5), (3, 8), (15, 4), (40, 3)])
def test_same_bits_on_every_run_and_guard_behind_the_workspace(m, g):
    p = Problem([(2500, m), (40, m), (1200, m)], 2, g, 16, HALF, E=400)
    need = rc.rc_cache_attend_workspace_size(p.cache, HALF, 3, 400, 2 * g, m)
    assert need > 0
    room = torch.full((need + 4096,), 0xa5, dtype=torch.uint8, device=DEV)
    first = p.run(workspace=room[:need])
    p.check(first)
    for _ in range(4):
        room[:need].random_(0, 256)
        r = p.run(workspace=room[:need])
        assert torch.equal(r["out"], first["out"]) and torch.equal(r["lse"], first["lse"])
    assert (room[need:] == 0xa5).all()


def test_another_stream_and_graph_replays():
    p = Problem([(2500, 1), (40, 1), (1200, 1)], 2, 5, 16, HALF, E=400)
    i = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    tables, ctx, starts = p.tables.to(DEV), i(p.ctx), i(p.starts)
    ids = p.tables[0, 0, :9].to(DEV)
    slot = torch.stack([p.slots[2499], p.slots[2539], p.slots[3739]]).to(DEV)
    k, v = p.k[:, :3].contiguous().to(DEV), p.v[:, :3].contiguous().to(DEV)
    ws = torch.empty(rc.rc_cache_attend_workspace_size(p.cache, HALF, 3, 400, 10, 1), dtype=torch.uint8, device=DEV)
    out, lse = torch.empty_like(p.q), torch.empty(p.q.shape[:3], device=DEV)
    blocks = [torch.empty((1, 9, 16, 2, 128), dtype=HALF, device=DEV) for _ in range(2)]

    def step():
        rc.rc_cache_write(k, v, slot, p.cache)
        rc.rc_cache_attend(p.q, p.cache, tables, ctx, starts, workspace=ws, out=out, lse=lse)
        rc.rc_cache_read(p.cache, ids, k=blocks[0], v=blocks[1])

    step()
    torch.cuda.synchronize()
    want = [t.clone() for t in (out, lse, *blocks)]
    other = torch.cuda.Stream()
    for t in (out, lse, *blocks):
        t.fill_(3)
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):
        step()
    torch.cuda.current_stream().wait_stream(other)
    assert all(torch.equal(a, b) for a, b in zip((out, lse, *blocks), want))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for replay in range(4):
        # new values and other lengths from one replay to the next, eager work in between
        k.copy_(torch.randn(k.shape, device=DEV))
        ctx.copy_(i([2500 - 300 * replay, 40, 1200]))
        for t in (out, lse, *blocks):
            t.fill_(float(replay))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (out, lse, *blocks)]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((out, lse, *blocks), got)), replay


@pytest.mark.parametrize("dtype", [HALF, BF])
def test_example_of_decoding_steps(dtype):
    """Write, attend, read back, search, remap, attend: the second request's sealed blocks go to the first one's, bit by bit the same."""
    from paper_2507_21433_amd import cache_example
    r = cache_example.main(dtype=dtype)
    assert r["matches"].tolist() == [[0, 1, 2, 3, 4]] and r["tables"][0, 1].tolist() == [0, 1, 2, 3, 4, 11] and r["freed"].sum() == 5
    assert torch.equal(r["before"]["out"], r["after"]["out"]) and torch.equal(r["before"]["lse"], r["after"]["lse"])
    assert torch.equal(r["after"]["out"][0, 0], r["after"]["out"][0, 1])
    assert torch.isfinite(r["prompt"]["out"]).all()

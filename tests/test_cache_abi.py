"""What the entry points of the 4-bit cache refuse, and what has nothing to do.  CPU only: every call fails validation or launches nothing."""
import ctypes
import os

import pytest
import torch

from paper_2507_21433_amd import binding as rc

FAKE, ODD = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1004)      # never dereferenced
OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
BLOCK = 8 * 2176


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(rc.LIB_PATH):
        from paper_2507_21433_amd import build
        build.build()
    return rc.lib()


def cdesc(L=2, T=16, H=8, D=128, dtype=0, n=10, stride=None):
    return rc.CacheDesc(L, T, H, D, dtype, n, n * H * (T // 16) * 2176 if stride is None else stride)


def write(lib, d, k=FAKE, v=FAKE, n=4, token=1024, layer=4096, slots=FAKE, cache=FAKE):
    return lib.rc_cache_write(d if d is None else ctypes.byref(d), k, v, n, token, layer, slots, cache, None)


def read(lib, d, cache=FAKE, ids=FAKE, n=4, kd=None, k=FAKE, v=FAKE):
    kd = rc.KvDesc(d.n_layers, d.block_tokens, d.n_kv_heads, 128, d.dtype, n * d.block_tokens * d.n_kv_heads * 128) if kd is None else kd
    return lib.rc_cache_read(ctypes.byref(d), cache, ids, n, ctypes.byref(kd), k, v, None)


def attend(lib, d, cache=FAKE, tables=FAKE, R=3, E=200, ctx=FAKE, start=FAKE, q=FAKE, n_q=3, heads=40, token=5120, layer=3 * 5120, max_q=1,
           scale=0.1, window=0, out=FAKE, lse=None, ws=FAKE, ws_bytes=1 << 30):
    return lib.rc_cache_attend(d if d is None else ctypes.byref(d), cache, tables, R, E, ctx, start, q, n_q, heads, token, layer, max_q, scale,
                               window, out, lse, ws, ws_bytes, None)


BAD_DESCS = [
    (None, INVALID), (cdesc(L=-1), INVALID), (cdesc(n=-1, stride=0), INVALID), (cdesc(T=8, stride=1 << 20), UNSUPPORTED),
    (cdesc(T=64), UNSUPPORTED), (cdesc(H=0), UNSUPPORTED), (cdesc(H=17), UNSUPPORTED), (cdesc(D=64), UNSUPPORTED),
    (cdesc(dtype=2), UNSUPPORTED), (cdesc(n=1 << 27, stride=1 << 50), UNSUPPORTED), (cdesc(stride=10 * BLOCK - 16), INVALID),
    (cdesc(stride=10 * BLOCK + 8), INVALID), (cdesc(L=65536), UNSUPPORTED),
]


@pytest.mark.parametrize("i", range(len(BAD_DESCS)))
def test_descriptors(lib, i):
    d, code = BAD_DESCS[i]
    assert write(lib, d) == code
    assert attend(lib, d) == code
    if d is not None:
        assert read(lib, d, kd=rc.KvDesc(2, 16, 8, 128, 0, 1 << 20)) == code
        assert lib.rc_cache_attend_workspace_size(ctypes.byref(d), 1, 200, 40, 1) == 0
    assert lib.rc_last_error()


def test_block_bytes(lib):
    assert lib.rc_cache_block_bytes(16, 8, 128) == BLOCK and lib.rc_cache_block_bytes(32, 3, 128) == 6 * 2176
    assert lib.rc_cache_block_bytes(24, 8, 128) == 0 and lib.rc_cache_block_bytes(16, 8, 64) == 0 and lib.rc_cache_block_bytes(16, 17, 128) == 0


def test_write_refusals(lib):
    d = cdesc()
    assert write(lib, d, n=0, k=None, v=None, slots=None, cache=None) == OK
    assert write(lib, cdesc(L=0), k=None) == OK and write(lib, cdesc(n=0), k=None) == OK
    for bad in (dict(k=None), dict(v=None), dict(slots=None), dict(cache=None), dict(k=ODD), dict(v=ODD), dict(cache=ODD), dict(n=-1),
                dict(token=1016), dict(token=1028), dict(layer=4100), dict(layer=1016), dict(layer=-8), dict(token=1 << 62)):
        assert write(lib, d, **bad) == INVALID, bad
    assert write(lib, d, n=1 << 40, token=1024) == UNSUPPORTED


def test_read_refusals(lib):
    d = cdesc()
    assert read(lib, d, n=0, cache=None, ids=None, k=None, v=None) == OK
    for bad in (dict(cache=None), dict(ids=None), dict(k=None), dict(v=None), dict(cache=ODD), dict(k=ODD), dict(v=ODD)):
        assert read(lib, d, **bad) == INVALID, bad
    for kd in (rc.KvDesc(1, 16, 8, 128, 0, 1 << 20), rc.KvDesc(2, 32, 8, 128, 0, 1 << 20), rc.KvDesc(2, 16, 4, 128, 0, 1 << 20),
               rc.KvDesc(2, 16, 8, 128, 1, 1 << 20), rc.KvDesc(2, 16, 8, 128, 0, 100)):
        assert read(lib, d, kd=kd) == INVALID
    assert read(lib, d, n=-1, kd=rc.KvDesc(2, 16, 8, 128, 0, 1 << 20)) == INVALID
    assert read(lib, d, n=1 << 30, kd=rc.KvDesc(2, 16, 8, 128, 0, 1 << 50)) == UNSUPPORTED


def test_attend_refusals(lib):
    d = cdesc()
    assert attend(lib, d, R=0) == OK and attend(lib, d, n_q=0) == OK and attend(lib, d, max_q=0) == OK and attend(lib, cdesc(L=0)) == OK
    for bad in (dict(cache=None), dict(tables=None), dict(ctx=None), dict(q=None), dict(out=None), dict(cache=ODD), dict(q=ODD), dict(out=ODD),
                dict(R=-1), dict(E=-1), dict(n_q=-1), dict(max_q=-1), dict(window=-1), dict(heads=0), dict(heads=41), dict(token=5112),
                dict(token=5124), dict(layer=5112), dict(layer=15364), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")),
                dict(scale=float("inf")), dict(start=None, max_q=2), dict(start=None, n_q=2), dict(token=1 << 62)):
        assert attend(lib, d, **bad) == INVALID, bad
    for bad in (dict(heads=2048, token=1 << 20, layer=1 << 30), dict(E=1 << 27), dict(n_q=1 << 31), dict(R=1 << 31)):
        assert attend(lib, d, **bad) == UNSUPPORTED, bad
    need = lib.rc_cache_attend_workspace_size(ctypes.byref(d), 3, 200, 40, 1)
    assert 0 < need < 72 << 20
    for bad in (dict(ws=None), dict(ws=ODD), dict(ws_bytes=need - 1)):
        assert attend(lib, d, **bad) == WORKSPACE, bad


def test_workspace_size_never_falls(lib):
    last = 0
    for R, E, heads, q in ((1, 8, 40, 1), (1, 200, 40, 1), (3, 200, 40, 1), (3, 20000, 40, 1), (3, 20000, 40, 3), (3, 20000, 40, 6),
                           (3, 20000, 40, 7), (64, 20000, 40, 1000), (64, 20000, 40, 100000)):
        sizes = [lib.rc_cache_attend_workspace_size(ctypes.byref(cdesc(L=L)), R, E, heads, q) for L in (1, 2, 64)]
        assert sizes == sorted(sizes) and sizes[0] >= last, (R, E, heads, q, sizes, last)
        last = sizes[0]
        assert sizes[-1] < 72 << 20
    # a step of fewer query tokens, of shorter tables or of fewer requests never needs more
    for q in (1, 2, 3, 6, 7, 50):
        assert lib.rc_cache_attend_workspace_size(ctypes.byref(cdesc()), 3, 200, 40, q) <= last


class Recorder:
    def __getattr__(self, name):
        return lambda *args: 16 if name.endswith("_size") else rc.RC_OK


@pytest.fixture
def library(monkeypatch):
    monkeypatch.setattr(rc, "lib", lambda: Recorder())
    monkeypatch.setattr(rc, "_dev", lambda *ts: None)
    monkeypatch.setattr(rc, "_stream", lambda: 0)


def test_binding_checks(library):
    half, bf = torch.float16, torch.bfloat16
    cache = rc.cache_tensor(2, 5, 16, 4, "cpu")
    kv = lambda *shape, dtype=half: torch.zeros(shape, dtype=dtype)
    slots, ids = torch.zeros(3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    rc.rc_cache_write(kv(2, 3, 4, 128), kv(2, 3, 4, 128), slots, cache)
    wide = kv(2, 3, 12, 128)
    rc.rc_cache_write(wide[:, :, 4:8], wide[:, :, 8:], slots, cache)
    for k, v, s, c in ((kv(1, 3, 4, 128), kv(1, 3, 4, 128), slots, cache), (kv(2, 3, 3, 128), kv(2, 3, 3, 128), slots, cache),
                       (kv(2, 3, 4, 128), kv(2, 3, 4, 128, dtype=bf), slots, cache), (kv(2, 3, 4, 128), kv(2, 4, 4, 128), slots, cache),
                       (kv(2, 3, 4, 128), wide[:, :, :4], slots, cache), (kv(2, 3, 4, 128), kv(2, 3, 4, 128), slots.long(), cache),
                       (kv(2, 3, 4, 128), kv(2, 3, 4, 128), slots[:2], cache), (kv(2, 3, 4, 128), kv(2, 3, 4, 128), slots, cache.char()),
                       (kv(2, 3, 4, 128), kv(2, 3, 4, 128), slots, cache[:, :, :, :, :2000]),
                       (kv(2, 3, 128, 4).transpose(2, 3), kv(2, 3, 128, 4).transpose(2, 3), slots, cache)):
        with pytest.raises(AssertionError):
            rc.rc_cache_write(k, v, s, c)
    with pytest.raises(TypeError):
        rc.rc_cache_write(kv(2, 3, 4, 128).float(), kv(2, 3, 4, 128).float(), slots, cache)
    rc.rc_cache_read(cache, ids, half)
    for kw in (dict(ids=ids.long()), dict(k=kv(2, 3, 16, 4, 128)), dict(k=kv(2, 2, 16, 4, 128), v=kv(2, 2, 16, 4, 128, dtype=bf))):
        with pytest.raises(AssertionError):
            rc.rc_cache_read(cache, kw.pop("ids", ids), half, **kw)
    tables, ctx, start = torch.zeros((2, 3, 7), dtype=torch.int32), torch.zeros(3, dtype=torch.int32), torch.zeros(4, dtype=torch.int32)
    q = kv(2, 5, 8, 128)
    r = rc.rc_cache_attend(q, cache, tables, ctx, start, max_q=2)
    assert r["out"].shape == q.shape and r["lse"].shape == (2, 5, 8)
    assert rc.rc_cache_attend(q, cache, tables, ctx, start, max_q=2, want_lse=False)["lse"] is None
    for kw in (dict(q=kv(1, 5, 8, 128)), dict(tables=tables[:1]), dict(tables=tables.long()), dict(tables=tables[:, :, ::2]), dict(ctx_len=ctx[:2]),
               dict(ctx_len=ctx.long()), dict(q_start=ctx), dict(out=kv(2, 5, 8, 128, dtype=bf)), dict(out=kv(2, 5, 16, 128)[:, :, ::2]),
               dict(lse=torch.zeros(2, 5, 8, dtype=half)), dict(lse=torch.zeros(2, 5, 4))):
        a = dict(dict(q=q, cache=cache, tables=tables, ctx_len=ctx, q_start=start, max_q=2), **kw)
        with pytest.raises(AssertionError):
            rc.rc_cache_attend(**a)


@pytest.mark.parametrize("H", [1, 2, 3, 8])
def test_workspace_size_never_falls_in_any_direction(lib, H):
    """A call with fewer query tokens than it announces is planned for these, an engine keeps one workspace for its largest step: no smaller call
    needs more."""
    tokens, requests, entries = (1, 2, 3, 4, 5, 6, 8, 10, 12, 16, 17, 20, 32, 33, 64, 65, 128, 300), (1, 2, 3, 5, 9, 20, 70), \
        list(range(60, 140, 3)) + [150, 250, 333, 512, 1000, 1023, 1025, 1200, 5000, 70000]
    for g in (1, 2, 3, 5, 8, 16):
        size = lambda q, R, E, L: lib.rc_cache_attend_workspace_size(ctypes.byref(rc.CacheDesc(L, 16, H, 128, 0, 100000, 100000 * H * 2176)), R, E, H * g, q)
        table = [[[size(q, R, E, 1) for E in entries] for R in requests] for q in tokens]
        for i, by_r in enumerate(table):
            for j, by_e in enumerate(by_r):
                assert by_e == sorted(by_e), (g, tokens[i], requests[j])
                assert i == 0 or all(a <= b for a, b in zip(table[i - 1][j], by_e)), (g, tokens[i], requests[j])
                assert j == 0 or all(a <= b for a, b in zip(by_r[j - 1], by_e)), (g, tokens[i], requests[j])
        assert all(size(q, R, E, 1) <= size(q, R, E, 4) for q in (1, 9, 65) for R in (1, 9) for E in entries)

"""What the entry points of the 16-bit blocks refuse, and what has nothing to do.  CPU only: every call fails validation or launches nothing."""
import ctypes
import os

import pytest
import torch

from paper_2507_21433_amd import binding as rc

FAKE, OTHER, ODD = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x2000), ctypes.c_void_p(0x1004)      # never dereferenced
OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
BLOCK = 16 * 8 * 128


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(rc.LIB_PATH):
        from paper_2507_21433_amd import build
        build.build()
    return rc.lib()


def desc(L=2, T=16, H=8, D=128, dtype=0, n=10, stride=None):
    return rc.KvDesc(L, T, H, D, dtype, n * T * H * 128 if stride is None else stride)


def by(d):
    return d if d is None else ctypes.byref(d)


def write(lib, d, blocks=10, k_new=FAKE, v_new=FAKE, n=4, token=1024, layer=4096, slots=FAKE, k=FAKE, v=FAKE):
    return lib.rc_kv_write(by(d), blocks, k_new, v_new, n, token, layer, slots, k, v, None)


def attend(lib, d, blocks=10, k=FAKE, v=FAKE, tables=FAKE, R=3, E=200, ctx=FAKE, start=FAKE, q=FAKE, n_q=3, heads=40, token=5120, layer=3 * 5120, max_q=1,
           scale=0.1, window=0, out=FAKE, lse=None, w_in=None, w_out=None, ws=FAKE, ws_bytes=1 << 30):
    return lib.rc_kv_attend(by(d), blocks, k, v, tables, R, E, ctx, start, q, n_q, heads, token, layer, max_q, scale, window, out, lse, w_in, w_out, ws,
                            ws_bytes, None)


def evict(lib, L=2, t_in=FAKE, t_out=FAKE, R=3, E=20, NB=10, T=16, ctx=FAKE, weights=FAKE, keep=FAKE, first=1, last=1, r_in=FAKE, r_out=FAKE, n=FAKE):
    return lib.rc_kv_evict(L, t_in, t_out, R, E, NB, T, ctx, weights, keep, first, last, r_in, r_out, n, None)


BAD = [
    (None, 10, INVALID), (desc(L=-1), 10, INVALID), (desc(), -1, INVALID), (desc(T=8, stride=1 << 20), 10, UNSUPPORTED), (desc(T=64), 10, UNSUPPORTED),
    (desc(H=0), 10, UNSUPPORTED), (desc(H=17), 10, UNSUPPORTED), (desc(D=64), 10, UNSUPPORTED), (desc(dtype=2), 10, UNSUPPORTED),
    (desc(stride=1 << 60), 1 << 27, UNSUPPORTED), (desc(stride=1 << 60), 1 << 62, UNSUPPORTED), (desc(T=32, stride=1 << 60), 1 << 26, UNSUPPORTED),
    (desc(), 11, INVALID), (desc(stride=10 * BLOCK + 4), 10, INVALID), (desc(L=65536), 10, UNSUPPORTED),
]


@pytest.mark.parametrize("i", range(len(BAD)))
def test_descriptors(lib, i):
    d, blocks, code = BAD[i]
    assert write(lib, d, blocks) == code
    assert attend(lib, d, blocks) == code
    assert lib.rc_kv_attend_workspace_size(by(d), blocks, 1, 200, 40, 1, 1, 0) == 0
    assert lib.rc_last_error()


def test_write_refusals(lib):
    d = desc()
    assert write(lib, d, n=0, k=None, v=None, slots=None, k_new=None) == OK
    assert write(lib, desc(L=0), k=None) == OK and write(lib, desc(n=0), 0, k=None) == OK
    for bad in (dict(k=None), dict(v=None), dict(slots=None), dict(k_new=None), dict(v_new=None), dict(k=ODD), dict(v=ODD), dict(k_new=ODD), dict(v_new=ODD),
                dict(n=-1), dict(token=1016), dict(token=1028), dict(layer=4100), dict(layer=1016), dict(layer=-8), dict(token=1 << 62)):
        assert write(lib, d, **bad) == INVALID, bad
    assert write(lib, d, n=1 << 40) == UNSUPPORTED and write(lib, d, n=1 << 25) == UNSUPPORTED


def test_attend_refusals(lib):
    d = desc()
    for nothing in (dict(R=0), dict(n_q=0), dict(max_q=0)):
        assert attend(lib, d, **nothing) == OK and attend(lib, d, w_in=FAKE, w_out=FAKE, **nothing) == OK
    assert attend(lib, desc(L=0)) == OK
    for bad in (dict(k=None), dict(v=None), dict(tables=None), dict(ctx=None), dict(q=None), dict(out=None), dict(k=ODD), dict(v=ODD), dict(q=ODD), dict(out=ODD),
                dict(R=-1), dict(E=-1), dict(n_q=-1), dict(max_q=-1), dict(window=-1), dict(heads=0), dict(heads=41), dict(token=5112),
                dict(token=5124), dict(layer=5112), dict(layer=15364), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")),
                dict(scale=float("inf")), dict(start=None, max_q=2), dict(start=None, n_q=2), dict(token=1 << 62), dict(w_in=FAKE)):
        assert attend(lib, d, **bad) == INVALID, bad
    for bad in (dict(heads=2048, token=1 << 20, layer=1 << 30), dict(E=1 << 27), dict(n_q=1 << 31), dict(R=1 << 31), dict(R=1 << 10, E=1 << 19, n_q=1 << 10, w_out=FAKE)):
        assert attend(lib, d, **bad) == UNSUPPORTED, bad
    for weigh in (0, 1):
        need = lib.rc_kv_attend_workspace_size(by(d), 10, 3, 200, 40, 3, 1, weigh)
        assert 0 < need < 80 << 20
        for bad in (dict(ws=None), dict(ws=ODD), dict(ws_bytes=need - 1)):
            assert attend(lib, d, w_out=FAKE if weigh else None, **bad) == WORKSPACE, bad


def test_evict_refusals(lib):
    assert evict(lib, L=0) == OK and evict(lib, R=0, NB=0) == OK
    for bad in (dict(L=-1), dict(R=-1), dict(E=-1), dict(NB=-1), dict(first=-1), dict(last=0), dict(last=-5), dict(t_in=None), dict(t_out=None), dict(ctx=None),
                dict(weights=None), dict(keep=None), dict(r_in=None), dict(r_out=None), dict(n=None)):
        assert evict(lib, **bad) == INVALID, bad
    for bad in (dict(T=8), dict(T=64), dict(E=1 << 31), dict(NB=1 << 31), dict(R=1 << 24), dict(R=1 << 60)):
        assert evict(lib, **bad) == UNSUPPORTED, bad


@pytest.mark.parametrize("H", [1, 3, 8])
def test_workspace_size_never_falls(lib, H):
    """An engine keeps one workspace for its largest step: no smaller call needs more, with weights no less than without."""
    tokens, requests, entries = (1, 2, 3, 4, 6, 8, 16, 17, 32, 33, 64, 300, 5000), (1, 2, 9, 70), [1, 60, 64, 65, 100, 128, 250, 1023, 1200, 5000, 70000]
    for g in (1, 2, 5, 8, 16, 40):
        size = lambda q, R, E, L, n, w: lib.rc_kv_attend_workspace_size(by(rc.KvDesc(L, 16, H, 128, 0, 1 << 40)), 100000, R, E, H * g, n, q, w)
        for w in (0, 1):
            table = [[[size(q, R, E, 1, R * q, w) for E in entries] for R in requests] for q in tokens]
            for i, by_r in enumerate(table):
                for j, by_e in enumerate(by_r):
                    assert by_e == sorted(by_e), (g, tokens[i], requests[j])
                    assert i == 0 or all(a <= b for a, b in zip(table[i - 1][j], by_e)), (g, tokens[i], requests[j])
                    assert j == 0 or all(a <= b for a, b in zip(by_r[j - 1], by_e)), (g, tokens[i], requests[j])
            assert all(size(q, R, E, 1, R * q, w) <= size(q, R, E, 4, R * q, w) for q in (1, 9, 65) for R in (1, 9) for E in entries)
            assert all(size(q, 9, 300, 1, n, w) <= size(q, 9, 300, 1, n + 100, w) for q in (1, 9, 65) for n in (9, 100, 5000))
        assert all(size(q, 9, E, 1, 9 * q, 0) <= size(q, 9, E, 1, 9 * q, 1) for q in tokens for E in entries)


@pytest.mark.parametrize("weigh", [False, True])
def test_the_workspace_that_is_asked_for_is_enough(lib, weigh):
    """For the largest step and for every smaller one: a call is refused for nothing else (a NULL workspace says what it would have needed)."""
    for H, g in ((1, 1), (2, 5), (8, 4), (4, 40)):
        d = rc.KvDesc(1, 32, H, 128, 1, 1 << 40)
        for R in (1, 7, 80):
            # (without weights tables of up to 1024 tokens need none: such a call would be launched)
            for E in (1, 40, 900, 30000) if weigh else (40, 900, 30000):
                for most in (1, 5, 9, 100, 4000):
                    have = lib.rc_kv_attend_workspace_size(by(d), 100000, R, E, H * g, R * most, most, int(weigh))
                    for q in {1, 3, 7, most // 2 + 1, most} - {x for x in (3, 7) if x > most}:
                        code = attend(lib, d, 100000, R=R, E=E, n_q=R * q, heads=H * g, token=H * g * 128, max_q=q, w_out=FAKE if weigh else None, ws=None)
                        assert code == WORKSPACE
                        need = int(lib.rc_last_error().split()[-4])
                        assert need <= have, (H, g, R, E, most, q)


class Recorder:
    def __getattr__(self, name):
        return lambda *args: 16 if name.endswith("_size") else rc.RC_OK


@pytest.fixture
def library(monkeypatch):
    monkeypatch.setattr(rc, "lib", lambda: Recorder())
    monkeypatch.setattr(rc, "_dev", lambda *ts: None)
    monkeypatch.setattr(rc, "_stream", lambda: 0)


half, bf = torch.float16, torch.bfloat16


def kv(*shape, dtype=half):
    return torch.zeros(shape, dtype=dtype)


def i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def test_binding_checks_of_write(library):
    k, v, slots = kv(2, 5, 16, 4, 128), kv(2, 5, 16, 4, 128), i32(3)
    rc.rc_kv_write(kv(2, 3, 4, 128), kv(2, 3, 4, 128), slots, k, v)
    wide = kv(2, 3, 12, 128)
    rc.rc_kv_write(wide[:, :, 4:8], wide[:, :, 8:], slots, k[:, 1:4], v[:, 1:4])
    x = kv(2, 3, 4, 128)
    for a in ((kv(1, 3, 4, 128), kv(1, 3, 4, 128), slots, k, v), (kv(2, 3, 3, 128), kv(2, 3, 3, 128), slots, k, v), (x, kv(2, 3, 4, 128, dtype=bf), slots, k, v),
              (x, kv(2, 4, 4, 128), slots, k, v), (x, wide[:, :, :4], slots, k, v), (x, x, slots.long(), k, v), (x, x, slots[:2], k, v),
              (x, x, slots, k.to(bf), v.to(bf)), (x, x, slots, k, v[:, :4]), (x, x, slots, k[:, ::2], v[:, ::2]), (x, x, slots, k, v[:1]),
              (x, x, slots, k[:, 1:4], kv(2, 3, 16, 4, 128)),
              (kv(2, 3, 128, 4).transpose(2, 3), kv(2, 3, 128, 4).transpose(2, 3), slots, k, v)):
        with pytest.raises(AssertionError):
            rc.rc_kv_write(*a)
    with pytest.raises(TypeError):
        rc.rc_kv_write(x.float(), x.float(), slots, k.float(), v.float())


def test_binding_checks_of_attend(library):
    k, v = kv(2, 5, 16, 4, 128), kv(2, 5, 16, 4, 128)
    tables, ctx, start, q = i32(2, 3, 7), i32(3), i32(4), kv(2, 5, 8, 128)
    r = rc.rc_kv_attend(q, k, v, tables, ctx, start, max_q=2)
    assert r["out"].shape == q.shape and r["lse"].shape == (2, 5, 8) and r["weights"] is None
    assert rc.rc_kv_attend(q, k, v, tables, ctx, start, max_q=2, want_lse=False)["lse"] is None
    w = torch.zeros(2, 3, 7)
    assert rc.rc_kv_attend(q, k, v, tables, ctx, start, want_weights=True)["weights"].shape == w.shape
    assert rc.rc_kv_attend(q, k, v, tables, ctx, start, weights_in=w)["weights"] is not w
    assert rc.rc_kv_attend(q, k, v, tables, ctx, start, weights_in=w, weights_out=w)["weights"] is w
    for kw in (dict(q=kv(1, 5, 8, 128)), dict(q=q.to(bf)), dict(v=v.to(bf)), dict(v=v[:, :4]), dict(k=k[:, ::2], v=v[:, ::2]), dict(tables=tables[:1]),
               dict(tables=tables.long()), dict(tables=tables[:, :, ::2]), dict(ctx_len=ctx[:2]), dict(ctx_len=ctx.long()), dict(q_start=ctx),
               dict(out=kv(2, 5, 8, 128, dtype=bf)), dict(out=kv(2, 5, 16, 128)[:, :, ::2]), dict(lse=torch.zeros(2, 5, 8, dtype=half)), dict(lse=torch.zeros(2, 5, 4)),
               dict(weights_in=w[:1]), dict(weights_out=w.double()), dict(weights_out=torch.zeros(2, 3, 14)[:, :, ::2]),
               dict(workspace=torch.zeros(64, dtype=torch.uint8)[::2])):
        a = dict(dict(q=q, k=k, v=v, tables=tables, ctx_len=ctx, q_start=start, max_q=2), **kw)
        with pytest.raises(AssertionError):
            rc.rc_kv_attend(**a)


def test_binding_checks_of_evict(library):
    a = dict(tables=i32(2, 3, 7), weights=torch.zeros(2, 3, 7), ctx_len=i32(3), keep=i32(3), refcount=i32(2, 9), block_tokens=16)
    r = rc.rc_kv_evict(**a)
    assert r["tables"] is not a["tables"] and r["n_evicted"].shape == (2, 3)
    r = rc.rc_kv_evict(**a, in_place=True)
    assert r["tables"] is a["tables"] and r["refcount"] is a["refcount"]
    out = dict(tables=i32(2, 3, 7), refcount=i32(2, 9), n_evicted=i32(2, 3))
    assert rc.rc_kv_evict(**a, out=out)["tables"] is out["tables"]
    for kw in (dict(tables=i32(2, 3, 7).long()), dict(tables=i32(2, 3, 14)[:, :, ::2]), dict(weights=torch.zeros(2, 3, 8)), dict(weights=torch.zeros(2, 3, 7).half()),
               dict(ctx_len=i32(2)), dict(keep=i32(4)), dict(keep=i32(3).long()), dict(refcount=i32(1, 9)), dict(refcount=i32(18)),
               dict(out=dict(out, tables=i32(2, 3, 8))), dict(out=dict(out, refcount=i32(2, 8))), dict(out=dict(out, n_evicted=i32(2))), dict(out=out, in_place=True)):
        with pytest.raises(AssertionError):
            rc.rc_kv_evict(**dict(a, **kw))

"""Arguments at the limits of the 4-bit cache's entry points.  CPU only: every call fails validation or launches nothing."""
import pytest
import torch

from paper_2507_21433_amd import binding as rc
from tests.test_cache_abi import INVALID, ODD, WORKSPACE, attend, cdesc, lib, library, read  # noqa: F401


@pytest.mark.parametrize("scale", [2.4e38, 2.9e38, 3.4e38])
def test_scale_whose_product_is_no_number(lib, scale):  # noqa: F811
    """Every exponent would be infinite or NaN."""
    assert attend(lib, cdesc(), scale=scale) == INVALID


@pytest.mark.parametrize("scale", [1e-45, 1.0, 2.3e38])
def test_scales_that_are_taken(lib, scale):  # noqa: F811
    # (as far as the workspace, which is missing)
    assert attend(lib, cdesc(), scale=scale, ws=None) == WORKSPACE


def test_max_q_left_out(monkeypatch):
    """One query token per request without starts; with starts as many as there are, so that none is left out."""
    seen = {}

    class Library:
        def __getattr__(self, name):
            def call(*args):
                seen[name] = args
                return 16 if name.endswith("_size") else rc.RC_OK
            return call

    monkeypatch.setattr(rc, "lib", lambda: Library())
    monkeypatch.setattr(rc, "_dev", lambda *ts: None)
    monkeypatch.setattr(rc, "_stream", lambda: 0)
    cache, tables = rc.cache_tensor(1, 5, 16, 2, "cpu"), torch.zeros((1, 3, 7), dtype=torch.int32)
    ctx, starts = torch.zeros(3, dtype=torch.int32), torch.tensor([0, 7, 7, 9], dtype=torch.int32)
    for N, kw, want in ((3, {}, 1), (9, dict(q_start=starts), 9), (9, dict(q_start=starts, max_q=7), 7)):
        rc.rc_cache_attend(torch.zeros((1, N, 4, 128), dtype=torch.float16), cache, tables, ctx, **kw)
        assert seen["rc_cache_attend"][12] == want and seen["rc_cache_attend_workspace_size"][4] == want, (N, kw)


def test_read_of_no_blocks_needs_no_cache(lib):  # noqa: F811
    """No address is asked for where there is nothing to read (the other pointers are asked for as ever)."""
    for missing in ("ids", "k", "v"):
        assert read(lib, cdesc(n=0), cache=None, **{missing: None}) == INVALID
        assert b"NULL" in lib.rc_last_error()
    assert read(lib, cdesc(n=0), cache=None, k=ODD) == INVALID and b"aligned" in lib.rc_last_error()
    assert read(lib, cdesc(n=1), cache=None) == INVALID and b"NULL" in lib.rc_last_error()


def test_workspace_of_less_memory_than_its_shape(library):  # noqa: F811
    """One byte seen a thousand times is not a thousand bytes to write to."""
    cache, tables = rc.cache_tensor(1, 5, 16, 2, "cpu"), torch.zeros((1, 3, 7), dtype=torch.int32)
    q, ctx, byte = torch.zeros((1, 3, 4, 128), dtype=torch.float16), torch.zeros(3, dtype=torch.int32), torch.zeros(1, dtype=torch.uint8)
    rc.rc_cache_attend(q, cache, tables, ctx, workspace=torch.zeros(1000, dtype=torch.uint8))
    for bad in (byte.expand(1 << 30), torch.zeros(64, dtype=torch.uint8)[::2]):
        with pytest.raises(AssertionError):
            rc.rc_cache_attend(q, cache, tables, ctx, workspace=bad)

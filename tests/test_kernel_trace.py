"""What the tests of dispatch make of a kernel trace that has lost events (CPU only: the profiler is replaced)."""
from types import SimpleNamespace

import pytest
import torch

from tests import paths
from tests.test_gpu_few import takes_few

NORMS, SHARES, SELECT, TILES = "rc::norms_block_kernel<false>", "rc::few_shares_kernel<false, 4>", "rc::few_select_kernel", "rc::match_tile_kernel<half, 256, 256, 0>"
COPY = "Memcpy DtoH (Device -> Host)"


def trace(kernels, times, lost=()):
    """Events of `times` calls that launch `kernels` and copy a result; `lost`: the numbers of launches whose kernels are missing."""
    events, n = [], 0
    for _ in range(times):
        for k in kernels:
            n += 1
            events.append(SimpleNamespace(name="hipLaunchKernel", id=n, device_type=torch.autograd.DeviceType.CPU))
            if n not in lost:
                events.append(SimpleNamespace(name=f"void {k}(char const*)", id=n, device_type=torch.autograd.DeviceType.CUDA))
        n += 1
        events.append(SimpleNamespace(name="hipMemcpyWithStream", id=n, device_type=torch.autograd.DeviceType.CPU))
        events.append(SimpleNamespace(name=COPY, id=n, device_type=torch.autograd.DeviceType.CUDA))
    return events


@pytest.fixture
def profiler(monkeypatch):
    """Sets what the profiler returns, trace by trace: functions of the number of calls that it covers; the last one again and again."""
    left, calls = [], []

    def set_traces(*traces):
        left[:] = traces
        return lambda: calls.append(0)

    class Profile:
        def __init__(self, **kw):
            pass

        def __enter__(self):
            calls.clear()
            return self

        def __exit__(self, *a):
            return False

        def events(self):
            return (left.pop(0) if len(left) > 1 else left[0])(len(calls))

    monkeypatch.setattr(torch.profiler, "profile", Profile)
    monkeypatch.setattr(torch.cuda, "synchronize", lambda: None)
    return set_traces


whole = lambda times: trace([NORMS, NORMS, SHARES, SELECT], times)


def test_two_whole_traces_are_enough(profiler):
    names = paths.kernel_names(profiler(whole, whole, lambda times: pytest.fail("a third trace")))
    assert sum(SHARES in n for n in names) == sum(SELECT in n for n in names) == 3


def test_kernels_without_their_events(profiler):
    # every launch of the search is recorded, and no kernel of it: the norms' alone, which lie in front
    lost = lambda times: trace([NORMS, NORMS, SHARES, SELECT], times, lost={5 * i + j for i in range(times) for j in (3, 4)})
    assert takes_few(profiler(lost, lost, whole))


def test_launches_lost_with_their_kernels(profiler):
    # the last call's are missing; every call's but one's; every call's
    cut = lambda times: trace([NORMS, NORMS, SHARES, SELECT], times)[:-4]
    one = lambda times: trace([NORMS, NORMS], times - 1) + trace([NORMS, NORMS, SHARES, SELECT], 1)
    every = lambda times: trace([NORMS, NORMS], times)
    for lost in (cut, one, every):
        for traces in ((lost, whole), (whole, lost, whole)):
            names = paths.kernel_names(profiler(*traces))
            assert sum(SHARES in n for n in names) == sum(SELECT in n for n in names) == sum(NORMS in n for n in names) // 2 > 0


def test_a_trace_that_is_never_whole_is_none(profiler):
    lost = lambda times: trace([NORMS, NORMS, SHARES, SELECT], times, lost={3})
    call = profiler(lost)
    assert paths.kernel_names(call) == [] and paths.tile_kernels(call) is None
    with pytest.raises(pytest.skip.Exception):
        takes_few(call)


def test_whole_traces_are_believed(profiler):
    # neither plan's kernels, both plans', other tiles than a test is about
    for kernels in ([NORMS, NORMS], [NORMS, SHARES, TILES]):
        with pytest.raises(AssertionError):
            takes_few(profiler(lambda times: trace(kernels, times)))


def test_other_tiles_than_the_wanted_ones(profiler):
    call = profiler(lambda times: trace([NORMS, TILES], times))
    assert not takes_few(call)
    paths.assert_tiles(call, (256, 256, 0))
    for want in ((256, 192, 0), (256, 256, 1)):
        with pytest.raises(AssertionError):
            paths.assert_tiles(call, want)
    with pytest.raises(AssertionError):
        paths.assert_tiles(call, (256, 256, 0), (256, 192, 3))

"""The library launches on the current device: tensors of another one are refused before anything is launched (CPU only, with stand-ins)."""
import pytest
import torch

from paper_2507_21433_amd import binding as rc


class Tensor:
    def __init__(self, device):
        self.device = device
        self.is_cuda = device >= 0

    def get_device(self):
        return self.device


@pytest.fixture(params=[0, 1])
def current(request, monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: request.param, raising=False)
    return request.param


def test_tensors_of_the_current_device(current):
    rc._dev(Tensor(current), None, Tensor(current))
    rc._dev(None)


def test_tensors_of_other_devices(current):
    other = 1 - current
    for ts in ((Tensor(other),), (Tensor(current), Tensor(other)), (Tensor(other), None, Tensor(current)), (Tensor(-1),), (Tensor(current), Tensor(-1))):
        with pytest.raises(AssertionError):
            rc._dev(*ts)


def test_host_tensors_where_there_is_no_gpu():
    with pytest.raises(AssertionError):
        rc._dev(torch.zeros(1))

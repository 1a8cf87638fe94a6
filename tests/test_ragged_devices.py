"""Products over ragged ranges: all tensors on one device, which is current when the kernels are launched.  The tensors of another
device are stand-ins that answer what the binding asks."""
import contextlib

import pytest
import torch

import paper_2202_09518_amd as nmf
from paper_2202_09518_amd import binding


class On:
    """A contiguous tensor on a device."""
    is_cuda = True

    def __init__(self, device, shape, dtype=torch.float32):
        self.device_index, self.shape, self.dtype = device, torch.Size(shape), dtype

    def get_device(self):
        return self.device_index

    def numel(self):
        return self.shape.numel()

    def element_size(self):
        return self.dtype.itemsize

    def stride(self):
        return torch.empty(self.shape, device="meta").stride()

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 256


@pytest.fixture
def entries(monkeypatch):
    """Current device, streams and C entries of a machine with two devices; records where each entry was called."""
    calls, current = [], [0]

    @contextlib.contextmanager
    def device(d):
        keep, current[0] = current[0], d
        yield
        current[0] = keep

    class Lib:
        def __getattr__(self, name):
            if name == "nmf_ragged_work_bytes":
                return lambda *args: 0
            return lambda *args: calls.append((name, current[0], args[-1])) or 0

    monkeypatch.setattr(binding, "_current_device", lambda: current[0])
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(binding, "_raw_stream", lambda d: 1000 + d)
    monkeypatch.setattr(binding, "lib", lambda: Lib())
    binding._need.cache_clear()
    yield calls
    binding._need.cache_clear()


def arguments(device):
    at = lambda *shape, dtype=torch.float32: On(device, shape, dtype)      # noqa: E731
    X, Y, B, off = at(4, 8), at(4, 6), at(2, 8, 6), at(3, dtype=torch.int64)
    run, koff, Wt, H = at(2, dtype=torch.int32), at(3, dtype=torch.int32), at(5, 8), at(5, 6)
    A, U, V, G, scale = at(8, 6), at(4, 3), at(4, 3), at(2, 8, 6), at(2)
    return {
        nmf.nmf_grouped_product: [X, off, 2, 4, B, False, 8, 6, Y],
        nmf.nmf_grouped_gradient: [X, Y, off, 2, 4, 8, 6, G],
        nmf.nmf_lowrank_product: [X, 4, A, False, 8, 6, off, run, 2, Wt, H, koff, 2, 3, scale, U, Y],
        nmf.nmf_lowrank_gradient: [X, Y, 4, 8, 6, off, run, 2, koff, 2, 3, U, V, Wt, H],
    }


@pytest.mark.parametrize("device", [0, 1])
def test_calls_run_on_the_device_of_their_tensors(device, entries):
    for call, args in arguments(device).items():
        call(*args)
        assert entries[-1] == (call.__name__, device, 1000 + device)


def test_tensors_of_two_devices_are_refused(entries):
    for call, args in arguments(1).items():
        for i, arg in enumerate(args):
            if isinstance(arg, On):
                args[i] = On(0, arg.shape, arg.dtype)
                with pytest.raises(ValueError):
                    call(*args)
                args[i] = arg
        with pytest.raises(ValueError):
            call(*args, work=On(0, (64,), torch.uint8))
    assert not entries

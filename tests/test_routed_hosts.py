"""Codes on the host: refused by the binding like any other tensor on the host, whichever operand it looks at first."""
import pytest
import torch

import paper_2202_09518_amd as nmf
from paper_2202_09518_amd import binding

E8 = torch.float8_e4m3fn


class OnDevice:
    """A contiguous tensor of device 0, for what the binding asks."""
    is_cuda = True

    def __init__(self, dtype, *shape):
        self.dtype, self.shape = dtype, torch.Size(shape)

    def get_device(self):
        return 0

    def stride(self):
        return torch.empty(self.shape, device="meta").stride()

    def numel(self):
        return self.shape.numel()

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 256


@pytest.fixture(autouse=True)
def device(monkeypatch):
    monkeypatch.setattr(binding, "_current_device", lambda: 0)
    monkeypatch.setattr(binding, "_stream_at", lambda d, stream: 0)


@pytest.mark.parametrize("codes", [E8, torch.uint8])
def test_product_of_codes_on_the_host(codes):
    x, xs = torch.zeros(4, 128, dtype=torch.uint8).view(codes), torch.zeros(4, 1)
    offsets = torch.zeros(2, dtype=torch.int64)
    B, bs, Y = OnDevice(codes, 1, 128, 128), OnDevice(torch.float32, 1, 1, 1), OnDevice(torch.bfloat16, 4, 128)
    with pytest.raises(ValueError, match="X8"):
        nmf.nmf_grouped_product8(x, xs, offsets, 1, 4, B, bs, False, 128, 128, Y)
    with pytest.raises(ValueError, match="B8"):
        nmf.nmf_grouped_product8(OnDevice(codes, 4, 128), OnDevice(torch.float32, 4, 1), OnDevice(torch.int64, 2), 1, 4,
                                 torch.zeros(1, 128, 128, dtype=torch.uint8).view(codes), bs, False, 128, 128, Y)


@pytest.mark.parametrize("dtype", [E8, torch.uint8, torch.bfloat16])
def test_rows_to_their_places_on_the_host(dtype):
    X, place = torch.zeros(4, 128, dtype=torch.uint8).to(dtype), torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError, match="X"):
        nmf.nmf_spread_rows(X, 4, 1, place, 128, X.clone(), scale=torch.zeros(4, 1), Yscale=torch.zeros(4, 1))

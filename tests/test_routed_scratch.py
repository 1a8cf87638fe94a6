"""Scratch that the 8-bit product asks for against what its calls make of it, by the arguments alone."""
import os
import re

import pytest
import torch

import paper_2202_09518_amd as nmf
from paper_2202_09518_amd import binding
from test_routed_far import ROOM, route

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LAYOUT = {False: getattr(nmf, "NMF_B_M_X_N", 0), True: getattr(nmf, "NMF_B_N_X_M", 0)}


def copied(rows, count, m, n, transposed, x, b):
    """Bytes of copies in rows of whole 16s, of the operands that are named."""
    up = lambda k: -(-k // 16) * 16
    return (rows * up(m) if x else 0) + (count * (n * up(m) if transposed else m * up(n)) if b else 0)


# rows, groups, m, n, transposed, operands whose copies are worth their time ("" where none is odd, None where they are not worth it)
CASES = [
    (2245, 22, 6197, 5568, False, "x"), (8192, 64, 4095, 4096, False, "x"), (512, 64, 4095, 2048, False, "x"), (2245, 22, 6197, 5568, True, None),
    (8192, 16, 4096, 4095, True, ""), (8192, 16, 4096, 4095, False, "b"), (8192, 16, 4095, 4096, True, "xb"), (8192, 1, 4096, 4096, True, ""),
    (8192, 1, 4096, 4096, False, ""), (6000, 4, 4095, 2047, False, "xb"), (6000, 4, 4095, 2047, True, "xb"), (20, 1, 100, 2 ** 22 + 5, True, None),
    (40000, 1, 4095, 2 ** 22 + 5, True, "xb"), (512, 64, 4096, 2047, False, None), (3, 1, 15, 15, False, None),
]


@pytest.mark.parametrize("rows,groups,m,n,transposed,odd", CASES)
def test_scratch_is_what_the_call_uses(rows, groups, m, n, transposed, odd):
    for typ in (nmf.NMF_F32, nmf.NMF_BF16):
        straight, copies, _, _, _, _, parts = route(typ, rows, groups, m, n, transposed)
        assert copies == copied(rows, groups, m, n, transposed, "x" in (odd or ""), "b" in (odd or "")) and straight == (odd is not None)
        need = nmf.nmf_routed_work_bytes(2 | LAYOUT[transposed], rows, m, n, groups)
        assert need == copies + parts
        if need:                                         # no byte less does
            assert route(typ, rows, groups, m, n, transposed, work=need)[1] == copies
            assert route(typ, rows, groups, m, n, transposed, work=need - 1)[1::5] != [copies, parts]
    both = [nmf.nmf_routed_work_bytes(2 | layout, rows, m, n, groups) for layout in LAYOUT.values()]
    assert nmf.nmf_routed_work_bytes(2, rows, m, n, groups) == max(both)


def test_scratch_of_operands_off_their_borders_and_far_apart():
    rows, groups, m, n = 8192, 16, 4096, 4096
    need = lambda kind, transposed: nmf.nmf_routed_work_bytes(2 | kind | LAYOUT[transposed], rows, m, n, groups)
    for transposed in (False, True):
        assert need(0, transposed) == 0
        assert need(nmf.NMF_ODD_X, transposed) == rows * m and need(nmf.NMF_ODD_B, transposed) == groups * m * n
        assert need(nmf.NMF_ODD_B | nmf.NMF_ONE_B, transposed) == m * n
        assert need(nmf.NMF_ODD_X, transposed) == route(nmf.NMF_BF16, rows, groups, m, n, transposed, ldx=2 ** 22)[1]
        assert need(nmf.NMF_ODD_B, transposed) == route(nmf.NMF_BF16, rows, groups, m, n, transposed, ldb=2 ** 22)[1]
        assert need(nmf.NMF_ODD_X, transposed) == route(nmf.NMF_BF16, rows, groups, m, n, transposed, first=1)[1]


def test_scratch_of_sizes_at_the_limits():
    most = 2 ** 31 - 1
    for kind in (2, 2 | nmf.NMF_ODD_X | nmf.NMF_ODD_B, 2 | LAYOUT[False], 2 | LAYOUT[True]):
        for m, n in ((most, most), (2 ** 22 - 17, most), (most, 2 ** 22 - 17), (2 ** 22 - 17, 2 ** 22 - 17)):
            assert 0 <= nmf.nmf_routed_work_bytes(kind, most, m, n, most) < 2 ** 63


def test_layouts_match_the_header():
    text = open(os.path.join(ROOT, "include", "nmfmu_routed.h")).read()
    for name in ("NMF_B_M_X_N", "NMF_B_N_X_M"):
        assert int(re.search(rf"{name} = (\d+)", text).group(1)) == getattr(nmf, name)
    assert ROOM > nmf.nmf_routed_work_bytes(2, 8192, 4095, 4095, 16)


class Codes:
    """A tensor of codes or of something else on the device, as the binding asks for it."""
    is_cuda = True

    def __init__(self, dtype, *shape, strides=None, at=256):
        self.dtype, self.shape, self.at = dtype, torch.Size(shape), at
        self.strides = strides or torch.empty(shape, device="meta").stride()

    def get_device(self):
        return 0

    def stride(self):
        return self.strides

    def numel(self):
        return self.shape.numel()

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return self.at


def test_the_binding_asks_for_what_the_call_uses(monkeypatch):
    asked = []
    monkeypatch.setattr(binding, "_current_device", lambda: 0)
    monkeypatch.setattr(binding, "_stream_at", lambda d, stream: 0)
    monkeypatch.setattr(binding, "_scratch", lambda need, work, d, stream: asked.append(need) or (None, 0, None))
    real = binding.lib()

    class Lib:
        nmf_routed_work_bytes, nmfmu_product8_route = real.nmf_routed_work_bytes, real.nmfmu_product8_route
        nmf_grouped_product8 = staticmethod(lambda *args: nmf.NMF_OK)

    monkeypatch.setattr(binding, "_lib", Lib)
    binding._need_routed.cache_clear()
    for rows, groups, m, n, transposed, odd in CASES:
        for pad in (0, 2 ** 22):
            E, F = torch.float8_e4m3fn, torch.float32
            r, c = (n, m) if transposed else (m, n)
            R, C = -(-r // 128), -(-c // 128)
            X = Codes(E, rows, m, strides=(m + pad, 1))
            nmf.nmf_grouped_product8(X, Codes(F, rows, -(-m // 128)), Codes(torch.int64, groups + 1), groups, rows, Codes(E, groups, r, c), Codes(F, groups, R, C), transposed,
                                     m, n, Codes(torch.bfloat16, rows, n))
            used = route(nmf.NMF_BF16, rows, groups, m, n, transposed, ldx=m + pad)
            assert asked.pop() == used[1] + used[6], (rows, groups, m, n, transposed, pad)

"""Operands of whole widths that lie off 16-byte borders by their base or leading dimension, as column slices do: they are copied like
those of odd widths, and the scratch has room for that.  Bounds as in test_ragged_products."""
import pytest
import torch

import paper_2202_09518_amd as nmf
from test_ragged_products import TYPES, Problem, within

gpu = pytest.mark.gpu


def test_scratch_has_room_for_copies_of_views():
    wb = nmf.nmf_ragged_work_bytes
    rows, m, n, e = 8192, 4096, 2048, 2
    plain = wb(0, nmf.NMF_BF16, rows, m, n, 3)
    assert wb(0 | nmf.NMF_ODD_X, nmf.NMF_BF16, rows, m, n, 3) == plain + rows * m * e
    assert wb(0 | nmf.NMF_ODD_B, nmf.NMF_BF16, rows, m, n, 3) == plain + 3 * m * n * e
    assert wb(0 | nmf.NMF_ODD_X | nmf.NMF_ODD_B, nmf.NMF_BF16, rows, m, n, 3) == plain + (rows * m + 3 * m * n) * e
    plain = wb(1, nmf.NMF_BF16, rows, m, n, 3)
    assert wb(1 | nmf.NMF_ODD_X, nmf.NMF_BF16, rows, m, n, 3) == plain + rows * m * e
    assert wb(1 | nmf.NMF_ODD_B, nmf.NMF_BF16, rows, m, n, 3) == plain + rows * n * e
    plain = wb(2, nmf.NMF_BF16, rows, m, n, 3, 2, 16, 32)
    assert wb(2 | nmf.NMF_ODD_X, nmf.NMF_BF16, rows, m, n, 3, 2, 16, 32) == plain + rows * m * e
    assert wb(2 | nmf.NMF_ODD_FACTORS, nmf.NMF_BF16, rows, m, n, 3, 2, 16, 32) == plain + 32 * (m + n) * e
    # widths that do not fill 16 bytes are in already; short products are not worth copies; other kinds are unknown
    assert wb(0 | nmf.NMF_ODD_X, nmf.NMF_BF16, rows, m - 1, n, 3) == wb(0, nmf.NMF_BF16, rows, m - 1, n, 3)
    assert wb(0 | nmf.NMF_ODD_X, nmf.NMF_BF16, 16, 256, 256, 1) == wb(0, nmf.NMF_BF16, 16, 256, 256, 1)
    assert wb(4 | nmf.NMF_ODD_X, nmf.NMF_BF16, rows, m, n, 3) == 0 and wb(256, nmf.NMF_BF16, rows, m, n, 3) == 0


@pytest.fixture
def scratch(monkeypatch):
    """Bytes of the scratch that the calls were given."""
    given, real = [], nmf.binding._work

    def work(*args):
        out = real(*args)
        given.append(out[1])
        return out

    monkeypatch.setattr(nmf.binding, "_work", work)
    return given


def sliced(rows, cols, dtype, g, odd, count=None):
    """A view one entry to the right in rows of cols + 8 entries."""
    mem = torch.randn(*(() if count is None else (count,)), rows, cols + 8, generator=g, device="cuda").to(dtype)
    return mem[..., 1:cols + 1] if odd else mem[..., :cols]


@gpu
@pytest.mark.parametrize("typ", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("odd_x,odd_b", [(True, False), (False, True), (True, True)])
def test_products_of_column_slices(odd_x, odd_b, transposed, typ, scratch):
    rows, groups, m, n = 2300, 2, 1024, 1536
    dt, e = TYPES[typ], 4 if typ == "f32" else 2
    g = torch.Generator(device="cuda").manual_seed(7)
    cut = [0, 900, rows]
    off = torch.tensor(cut, device="cuda")
    X, dY = sliced(rows, m, dt, g, odd_x), sliced(rows, n, dt, g, odd_b)
    B = sliced(*((n, m) if transposed else (m, n)), dt, g, odd_b, groups)
    Y, G = torch.empty(rows, n, dtype=dt, device="cuda"), torch.empty(groups, m, n, dtype=dt, device="cuda")
    nmf.nmf_grouped_product(X, off, groups, rows, B, transposed, m, n, Y)
    assert scratch[-1] >= (rows * m * e if odd_x else 0) + (groups * m * n * e if odd_b else 0)
    nmf.nmf_grouped_gradient(X, dY, off, groups, rows, m, n, G)
    assert scratch[-1] >= (rows * m * e if odd_x else 0) + (rows * n * e if odd_b else 0)
    for i in range(groups):
        x, w, dy = X[cut[i]:cut[i + 1]].double(), B[i].double(), dY[cut[i]:cut[i + 1]].double()
        w = w.t().contiguous() if transposed else w
        within(Y[cut[i]:cut[i + 1]], x @ w, x.abs() @ w.abs(), m, typ)
        within(G[i], x.t() @ dy, x.abs().t() @ dy.abs(), len(x), typ)


@gpu
@pytest.mark.parametrize("typ", ["f32", "bf16", "f16"])
def test_lowrank_products_of_column_slices(typ, scratch):
    rows, m, n = 2500, 1024, 1536
    dt, e = TYPES[typ], 4 if typ == "f32" else 2
    g = torch.Generator(device="cuda").manual_seed(8)
    p = Problem(rows, 5, 3, 4, 40, m, n, False, typ)
    p.X, p.A = sliced(rows, m, dt, g, True), sliced(m, n, dt, g, True)
    for name in ("Wt", "H"):                                   # contiguous, off the borders by their base alone
        t = getattr(p, name)
        mem = torch.empty(t.numel() + 1, dtype=dt, device="cuda")
        mem[1:].copy_(t.reshape(-1))
        setattr(p, name, mem[1:].view(t.shape))
    Y = torch.empty(rows, n, dtype=dt, device="cuda")
    p.forward(Y)
    assert scratch[-1] >= (rows * m + m * n + p.ktotal * (m + n)) * e
    p.check_product(Y, p.X.double(), p.A.double(), p.Wt.double(), p.H.double(), p.U)


@gpu
@pytest.mark.parametrize("transposed", [False, True])
def test_one_odd_matrix_for_many_groups_is_copied_once(transposed, scratch):
    rows, groups, m, n = 2300, 40, 1023, 1537
    g = torch.Generator(device="cuda").manual_seed(9)
    cut = [rows * i // groups for i in range(groups + 1)]
    X = torch.randn(rows, m, generator=g, device="cuda").bfloat16()
    B = torch.randn(*((n, m) if transposed else (m, n)), generator=g, device="cuda").bfloat16()
    Y = torch.empty(rows, n, dtype=torch.bfloat16, device="cuda")
    nmf.nmf_grouped_product(X, torch.tensor(cut, device="cuda"), groups, rows, B.expand(groups, *B.shape), transposed, m, n, Y)
    one = (rows * 1024 + 1024 * 1544) * 2                      # X and B in whole rows
    assert one - 2 * 1544 * 2 <= scratch[-1] < 2 * one
    x, w = X.double(), B.double()
    w = w.t().contiguous() if transposed else w
    within(Y, x @ w, x.abs() @ w.abs(), m, "bf16")

"""How many bits of U and V the products over ragged ranges keep.  Bounds as in test_ragged_products: an output in bf16 or f16 is off by
half a unit of its last place, a sum of K products held in fp32 by K 2^-23 of its magnitudes."""
import pytest
import torch

import paper_2202_09518_amd as nmf
from test_ragged_products import TYPES, within

gpu = pytest.mark.gpu


@gpu
@pytest.mark.parametrize("typ", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("kmax,scratch", [(16, True), (70, True), (16, False)])
def test_gradients_of_factors_keep_all_bits_of_u_and_v(kmax, scratch, typ):
    """Each run has two rows whose X and dY are equal and whose U and V nearly cancel: what is left of the sum of two products is
    2^-12 of them, and the sum may be off by two additions' roundings only, so 16 or 17 bits of U and V would show."""
    runs, m, n = 9, 136, 264
    rows = 2 * runs
    g = torch.Generator(device="cuda").manual_seed(kmax)
    dt = TYPES[typ]
    X = torch.randn(runs, m, generator=g, device="cuda").to(dt).repeat_interleave(2, 0).contiguous()
    dY = torch.randn(runs, n, generator=g, device="cuda").to(dt).repeat_interleave(2, 0).contiguous()

    def nearly_opposite():
        a = torch.randn(runs, 1, kmax, generator=g, device="cuda")
        b = -a * (1 + 2.0 ** -12 * torch.randn(runs, 1, kmax, generator=g, device="cuda"))
        return torch.cat([a, b], 1).reshape(rows, kmax).contiguous()

    U, V = nearly_opposite(), nearly_opposite()
    offsets = torch.arange(0, rows + 1, 2, device="cuda")
    run = torch.arange(runs, dtype=torch.int32, device="cuda")
    koff = (torch.arange(runs + 1, device="cuda") * kmax).int()
    dWt = torch.empty(runs * kmax, m, dtype=dt, device="cuda")
    dH = torch.empty(runs * kmax, n, dtype=dt, device="cuda")
    work = None if scratch else torch.empty(0, dtype=torch.uint8, device="cuda")
    nmf.nmf_lowrank_gradient(X, dY, rows, m, n, offsets, run, runs, koff, runs, kmax, U, V, dWt, dH, work=work)
    for r in range(runs):
        two, k = slice(2 * r, 2 * r + 2), slice(r * kmax, (r + 1) * kmax)
        for got, fac, mat in ((dWt, V, X), (dH, U, dY)):
            f, x = fac[two].double().t().contiguous(), mat[two].double()
            within(got[k], f @ x, f.abs() @ x.abs(), 2, typ)


@gpu
@pytest.mark.parametrize("typ", ["f16", "bf16"])
@pytest.mark.parametrize("spread", [8, 20, 26])
def test_products_of_factors_scaled_against_each_other(spread, typ):
    """Columns of W scaled by powers of two and rows of H by their inverses: the same product, so small entries of U count as much
    as large ones.  Pieces: bf16 2^-17 of each term; f16 2^-22 of it, and 2^-39 of the row's largest entry times H."""
    rows, m, n, k = 700, 64, 320, 6
    g = torch.Generator(device="cuda").manual_seed(spread)
    dt = TYPES[typ]
    by = 2.0 ** (spread // 2) * torch.ones(k, 1, device="cuda")
    by[1::2] = 2.0 ** -(spread - spread // 2)
    X = torch.randn(rows, m, generator=g, device="cuda").to(dt)
    Wt = (torch.randn(k, m, generator=g, device="cuda") / 8 * by).to(dt)
    H = (torch.randn(k, n, generator=g, device="cuda") / by).to(dt)
    A = torch.zeros(m, n, dtype=dt, device="cuda")
    U = torch.empty(rows, k, device="cuda")
    Y = torch.empty(rows, n, dtype=dt, device="cuda")
    offsets = torch.tensor([0, 300, rows], device="cuda")
    run = torch.zeros(2, dtype=torch.int32, device="cuda")
    koff = torch.tensor([0, k], dtype=torch.int32, device="cuda")
    nmf.nmf_lowrank_product(X, rows, A, False, m, n, offsets, run, 2, Wt, H, koff, 1, k, None, U, Y)
    x, w, h = X.double(), Wt.double().t().contiguous(), H.double()
    u = x @ w
    size = x.abs() @ w.abs() @ h.abs()
    if typ == "f16":
        pieces = 2.0 ** -22 * u.abs() @ h.abs() + 2.0 ** -39 * u.abs().amax(1, keepdim=True) * h.abs().sum(0)
    else:
        pieces = 2.0 ** -17 * u.abs() @ h.abs()
    within(Y, u @ h, size, m + k + 2, typ, pieces)

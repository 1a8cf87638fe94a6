"""Products over ragged ranges with rows that do not fill 16 bytes, large enough that operands are copied into whole rows first,
and more runs and segments than a wave has lanes.  Bounds as in test_ragged_products."""
import numpy as np
import pytest
import torch

import paper_2202_09518_amd as nmf
from test_ragged_products import TYPES, Problem, lengths_of, padded, result, untouched, within

gpu = pytest.mark.gpu


@gpu
@pytest.mark.parametrize("typ", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("rows,groups,m,n", [(2500, 3, 1023, 2049), (2048, 1, 1500, 1501), (2047, 1, 1001, 2048)])
def test_grouped_products_and_gradients_of_odd_rows(rows, groups, m, n, transposed, typ):
    assert nmf.nmf_ragged_work_bytes(0, nmf.NMF_BF16, rows, m, n, groups) > rows * m * 2          # room for a copy
    g = torch.Generator(device="cuda").manual_seed(rows)
    dt = TYPES[typ]
    cut = lengths_of("ragged", rows, groups, 5)
    off = torch.from_numpy(cut).cuda()
    X, _ = padded(rows, m, dt, g, 3, 1)
    dY, _ = padded(rows, n, dt, g, 2, 1)
    B = torch.randn(groups, *((n, m) if transposed else (m, n)), generator=g, device="cuda").to(dt)
    Y, mem = result(rows, n, dt, 1, 1)
    nmf.nmf_grouped_product(X, off, groups, rows, B, transposed, m, n, Y)
    G = torch.empty(groups, m, n, dtype=dt, device="cuda")
    nmf.nmf_grouped_gradient(X, dY, off, groups, rows, m, n, G)
    torch.cuda.synchronize()
    untouched(mem, Y, 1, 1)
    for i in range(groups):
        x, w, dy = X[cut[i]:cut[i + 1]].double(), B[i].double(), dY[cut[i]:cut[i + 1]].double()
        w = w.t().contiguous() if transposed else w
        within(Y[cut[i]:cut[i + 1]], x @ w, x.abs() @ w.abs(), m, typ)
        within(G[i], x.t() @ dy, x.abs().t() @ dy.abs(), max(1, len(x)), typ)


@gpu
@pytest.mark.parametrize("typ", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,segments,runs,kmin,kmax,m,n,transposed", [
    (2500, 9, 4, 5, 70, 1023, 1501, False), (2500, 9, 4, 5, 33, 1500, 1023, True),
    (1200, 150, 80, 1, 8, 264, 200, False), (2000, 70, 130, 2, 9, 128, 264, True),
])
def test_lowrank_of_odd_rows_and_many_runs(rows, segments, runs, kmin, kmax, m, n, transposed, typ):
    p = Problem(rows, segments, runs, kmin, kmax, m, n, transposed, typ)
    X, dY, A = p.X.double(), p.dY.double(), p.A.double()
    A = A.t().contiguous() if transposed else A
    W, H = p.Wt.double(), p.H.double()
    Y, ymem = result(rows, n, TYPES[typ], p.pad, p.first)
    dX, xmem = result(rows, m, TYPES[typ], p.pad, p.first)
    dWt, dH = torch.full_like(p.Wt, 5.0), torch.full_like(p.H, 5.0)
    p.forward(Y)
    p.backward(dX, dWt, dH)
    torch.cuda.synchronize()
    untouched(ymem, Y, p.pad, p.first)
    untouched(xmem, dX, p.pad, p.first)
    p.check_product(Y, X, A, W, H, p.U)
    p.check_product(dX, dY, A.t().contiguous(), H, W, p.V)
    p.check_gradient(dWt, dH)


@gpu
@pytest.mark.parametrize("typ", ["f32", "bf16", "f16"])
def test_factors_beside_ones_that_are_not_finite(typ):
    """Rows of H that follow each other in memory belong to different runs; with an odd width a chunk of 16 bytes holds both."""
    rows, m, n = 600, 200, 4101
    p = Problem(rows, 3, 3, 3, 5, m, n, False, typ, none=False)
    p.which = np.arange(3)
    p.run = torch.arange(3, dtype=torch.int32, device="cuda")
    Y, Z = (torch.empty(rows, n, dtype=TYPES[typ], device="cuda") for _ in range(2))
    for work in (None, torch.empty(4 * rows * 64, dtype=torch.uint8, device="cuda")):
        p.forward(Y, work)
        keep = p.H.clone()
        p.H[int(p.ko[1]):int(p.ko[2])] = float("inf")
        p.forward(Z, work)
        p.H.copy_(keep)
        torch.cuda.synchronize()
        clean = torch.ones(rows, dtype=torch.bool, device="cuda")
        clean[int(p.cut[1]):int(p.cut[2])] = False
        assert torch.equal(Y[clean], Z[clean])
        assert not bool(torch.isfinite(Z[~clean].float()).any())


@gpu
def test_range_of_u_in_f16():
    """U = X W_r beyond the range of f16 meets factors that bring the result back into it, and U far below that range likewise."""
    rows, m, n = 700, 64, 320
    p = Problem(rows, 4, 2, 4, 6, m, n, True, "f16", none=False)
    for up in (2.0 ** 13, 2.0 ** -12):
        p.X.copy_(torch.randn(rows, m, device="cuda"))
        p.Wt.copy_((torch.randn(p.ktotal, m, device="cuda") * up).half())
        p.scale.fill_(up)
        p.H.copy_((torch.randn(p.ktotal, n, device="cuda") * 2.0 ** -14).half() if up > 1 else (torch.randn(p.ktotal, n, device="cuda") * 2.0 ** 10).half())
        p.A.zero_()
        Y = torch.empty(rows, n, dtype=torch.float16, device="cuda")
        p.forward(Y)
        want = torch.zeros(rows, n, dtype=torch.float64, device="cuda")
        size = torch.zeros_like(want)
        for r, k, s in p.parts():
            u = p.X[r].double() @ p.Wt[k].double().t() * s
            want[r] = u @ p.H[k].double()
            size[r] = (p.X[r].double().abs() @ p.Wt[k].double().abs().t() * s) @ p.H[k].double().abs()
        fits = want.abs() < 60000
        got = torch.where(fits, Y.double(), 0.0)
        # pieces of u under its row's scale: 2^-22 of the row's largest entry for each of at most six factors; size bounds that
        within(got, torch.where(fits, want, 0.0), size, m + 8, "f16", 2.0 ** -17 * size)
        assert bool(torch.isfinite(Y[fits].float()).all())


@gpu
@pytest.mark.parametrize("typ", ["f32", "bf16"])
@pytest.mark.parametrize("rows,segments,runs,kmin,kmax,m,n", [
    (1500, 120, 5, 2, 20, 72, 8192),       # short segments beside a product of large tiles
    (300, 20, 300, 250, 256, 64, 64),      # more factors than a launch dimension holds
])
def test_short_segments_in_large_tiles_and_many_factors(rows, segments, runs, kmin, kmax, m, n, typ):
    p = Problem(rows, segments, runs, kmin, kmax, m, n, True, typ)
    X, dY, A = p.X.double(), p.dY.double(), p.A.double().t().contiguous()
    W, H = p.Wt.double(), p.H.double()
    Y, dX = torch.empty(rows, n, dtype=TYPES[typ], device="cuda"), torch.empty(rows, m, dtype=TYPES[typ], device="cuda")
    dWt, dH = torch.full_like(p.Wt, 5.0), torch.full_like(p.H, 5.0)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    p.forward(Y, stream=side)              # scratch of a stream that is not the current one
    side.synchronize()
    p.backward(dX, dWt, dH)
    torch.cuda.synchronize()
    p.check_product(Y, X, A, W, H, p.U)
    p.check_product(dX, dY, A.t().contiguous(), H, W, p.V)
    p.check_gradient(dWt, dH)

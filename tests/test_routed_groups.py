"""Routing and products in 8 bits against their definitions in 64 bits.

Bounds: a float operation loses at most 2^-24 of its result, exp at most 2^-22 (its own last places and the rounding of its
argument, of a magnitude below 128, which a factor of exp carries: |x| 2^-24); sums of n terms n 2^-24 of their magnitudes.
Products of codes whose results are in 16 bits: of eight neighbouring terms each loses less than 2^-13 of the largest one's power
of two, so a sum loses less than 7 2^-13 of the sum of the magnitudes; the root mean square of what is lost is much smaller, as
it has either sign, and is held to 2^-14 of the results'.
"""
import math

import pytest
import torch

import paper_2202_09518_amd as nmf

gpu = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
E8 = torch.float8_e4m3fn
U = 2.0 ** -24


def near(got, want, typ, lost):
    off, bound = (got.double() - want).abs(), HALF[typ] * (want.abs() + lost) + lost + (2.0 ** -25 if typ == "f16" else 0.0) + 2.0 ** -149
    bad = ~(off <= bound)
    assert not bool(bad.any()), (int(bad.sum()), float((off / bound).nan_to_num(1e30).max()))


def normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


# ---- products in 8 bits ------------------------------------------------------------------------

def codes(g, *shape):
    return (60 * normal(g, *shape)).clamp(-448, 448).to(E8)


def strided(t, pad, first):
    """The same values with rows `pad` entries apart, `first` entries into memory."""
    count, rows, cols = t.shape
    mem = torch.empty((rows + 1) * (cols + pad) * count + first, dtype=t.dtype, device="cuda").view(torch.uint8 if t.element_size() == 1 else t.dtype)
    v = mem.as_strided(t.shape, ((rows + 1) * (cols + pad), cols + pad, 1), first)
    v.copy_(t.view(v.dtype))
    return v.view(t.dtype) if v.is_contiguous() else v


def cuts(kind, rows, groups, seed):
    g = torch.Generator().manual_seed(seed)
    if kind == "even":
        return torch.linspace(0, rows, groups + 1).long()
    if kind == "one":                                        # all rows in one group, empty ones around it
        return torch.tensor([0] * (groups // 2 + 1) + [rows] * (groups - groups // 2))
    if kind == "inner":                                      # rows before and behind all groups
        return torch.linspace(rows // 4, rows - rows // 4, groups + 1).long()
    return torch.cat([torch.tensor([0]), torch.randint(0, rows + 1, (groups - 1,), generator=g).sort().values, torch.tensor([rows])])


def product(X, xs, B, bs, cut, transposed):
    """The sums in 64 bits, and those of the magnitudes."""
    rows, m = X.shape
    x = X.float().double() * xs.double().repeat_interleave(128, 1)[:, :m]
    n = B.shape[1] if transposed else B.shape[2]
    want, size = torch.zeros(rows, n, dtype=torch.float64, device="cuda"), torch.zeros(rows, n, dtype=torch.float64, device="cuda")
    for g in range(len(cut) - 1):
        a, b = int(cut[g]), int(cut[g + 1])
        if a < b:
            w = B[g].float().double() * bs[g].double().repeat_interleave(128, 0)[:B.shape[1]].repeat_interleave(128, 1)[:, :B.shape[2]]
            w = w.t().contiguous() if transposed else w
            want[a:b], size[a:b] = x[a:b] @ w, x[a:b].abs() @ w.abs()
    return want, size


def holds(Y, want, size, m, typ, ins):
    lost = ((m + 4) * U + (0 if typ == "f32" else 7 * 2.0 ** -13)) * size
    near(Y[ins], want[ins], typ, lost[ins])
    if typ != "f32" and bool(ins.any()):
        off = (Y[ins].double() - want[ins]).norm()
        assert float(off) <= float(want[ins].norm()) * (HALF[typ] + 2.0 ** -14) + 2.0 ** -25 * want[ins].numel() ** 0.5


PRODUCTS = [
    # rows, groups, m, n, lengths: one row, one column, widths below and beyond a block, every tile shape, parts of the contraction
    (1, 1, 1, 1, "even"), (1, 3, 128, 16, "one"), (5, 4, 7, 3, "ragged"), (33, 5, 130, 65, "ragged"), (40, 70, 96, 144, "ragged"),
    (24, 16, 2048, 256, "ragged"), (200, 3, 257, 129, "ragged"), (300, 2, 1024, 528, "ragged"), (130, 1, 4096, 272, "even"),
    (700, 9, 64, 384, "one"), (3400, 1, 208, 4112, "even"), (3400, 3, 80, 4096, "ragged"), (600, 5, 640, 640, "inner"),
    (2, 1, 16400, 200, "even"), (90, 2, 9000, 40, "ragged"),
]


@gpu
@pytest.mark.parametrize("typ", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("rows,groups,m,n,kind", PRODUCTS)
def test_grouped_product8(rows, groups, m, n, kind, transposed, typ):
    g = torch.Generator(device="cuda").manual_seed(rows + m)
    dt, cut = TYPES[typ], cuts(kind, rows, groups, rows)
    M, N = -(-m // 128), -(-n // 128)
    shape, blocks = ((n, m), (N, M)) if transposed else ((m, n), (M, N))
    off = cut.cuda()
    inside = torch.zeros(rows, dtype=torch.bool, device="cuda")
    inside[int(cut[0]):int(cut[-1])] = True
    x, b = codes(g, 1, rows, m), codes(g, groups, *shape)
    up = 2.0 ** -6 / m ** 0.5                                # results of about one, inside f16's range
    xs = torch.exp(normal(g, 1, rows, M)) * up
    bs = torch.exp(normal(g, groups, *blocks)) / 60
    want, size = product(x[0], xs[0], b, bs, cut, transposed)
    for pad, first in ((0, 0), (16, 32), (1, 3)):
        X, B, XS, BS = strided(x, pad, first)[0], strided(b, pad, first), strided(xs, pad, 0)[0], strided(bs, pad, 0)
        for work in (None, torch.empty(0, dtype=torch.uint8, device="cuda")):
            mem = torch.full(((rows + 1) * (n + pad) + first,), 77.0, device="cuda").to(dt)
            Y = mem.as_strided((rows, n), (n + pad, 1), first)
            nmf.nmf_grouped_product8(X, XS, off, groups, rows, B, BS, transposed, m, n, Y, work=work)
            torch.cuda.synchronize()
            holds(Y, want, size, m, typ, inside)
            keep = mem.clone()
            keep.as_strided((rows, n), (n + pad, 1), first)[inside] = 77.0
            assert bool((keep == torch.tensor(77.0).to(dt).item()).all())


@gpu
@pytest.mark.parametrize("typ", ["f32", "bf16"])
@pytest.mark.parametrize("transposed", [False, True])
def test_product8_of_large_tiles_and_its_gradient(transposed, typ):
    """The 256 x 256 tile, ragged at every edge; and dX = dY B^T as the call with B in its other form."""
    g = torch.Generator(device="cuda").manual_seed(11)
    rows, groups, m, n, dt = 5000, 3, 1040, 2064, TYPES[typ]
    cut = torch.tensor([0, 1801, 1803, 4990])
    inside = torch.arange(rows, device="cuda") < 4990
    shape = (n, m) if transposed else (m, n)
    B, BS = torch.empty(groups, *shape, dtype=E8, device="cuda"), torch.empty(groups, -(-shape[0] // 128), -(-shape[1] // 128), device="cuda")
    nmf.nmf_round_blocks(normal(g, groups, *shape), shape[0], shape[1], 128, B, BS)
    for k, cols, turned in ((m, n, transposed), (n, m, not transposed)):
        X, XS = torch.empty(rows, k, dtype=E8, device="cuda"), torch.empty(rows, -(-k // 128), device="cuda")
        nmf.nmf_round_blocks(normal(g, rows, k) / k ** 0.5, rows, k, 1, X, XS)
        Y = torch.full((rows, cols), 77.0, dtype=dt, device="cuda")
        nmf.nmf_grouped_product8(X, XS, cut.cuda(), groups, rows, B, BS, turned, k, cols, Y)
        want, size = product(X, XS, B, BS, cut, turned)
        holds(Y, want, size, k, typ, inside)
        assert bool((Y[~inside] == 77).all())


@gpu
def test_product8_of_one_matrix_for_all_groups_and_malformed_offsets():
    g = torch.Generator(device="cuda").manual_seed(12)
    rows, groups, m, n = 100, 4, 256, 144
    x, b = codes(g, 1, rows, m)[0], codes(g, 1, m, n)
    xs, bs = torch.rand(rows, 2, generator=g, device="cuda"), torch.rand(1, 2, 2, generator=g, device="cuda")
    cut = torch.tensor([0, 10, 10, 60, 100])
    Y, Z = torch.empty(rows, n, device="cuda"), torch.empty(rows, n, device="cuda")
    nmf.nmf_grouped_product8(x, xs, cut.cuda(), groups, rows, b.expand(groups, m, n), bs.expand(groups, 2, 2), False, m, n, Y)
    nmf.nmf_grouped_product8(x, xs, torch.tensor([0, 100]).cuda(), 1, rows, b, bs, False, m, n, Z)
    want, size = product(x, xs, b, bs, torch.tensor([0, 100]), False)
    ins = torch.ones(rows, dtype=torch.bool, device="cuda")
    holds(Y, want, size, m, "f32", ins)
    holds(Z, want, size, m, "f32", ins)
    mem = torch.full((rows + 64, n), 77.0, device="cuda")
    for bad in ([-5, 50, 20, 1000, 90], [2 ** 40, 0, 0, 100, 2 ** 62], [0, 100, 100, 100, 100000]):
        nmf.nmf_grouped_product8(x, xs, torch.tensor(bad).cuda(), groups, rows, b.expand(groups, m, n), bs.expand(groups, 2, 2), False, m, n, mem[:rows])
        torch.cuda.synchronize()
        assert bool((mem[rows:] == 77).all())


@gpu
@pytest.mark.parametrize("typ", ["f32", "bf16"])
@pytest.mark.parametrize("rows,n", [(3, 64), (50, 200), (400, 300), (3000, 2048)])
def test_product8_rows_and_columns_stand_alone(rows, n, typ):
    g = torch.Generator(device="cuda").manual_seed(13)
    m, groups = 400, 2
    cut = torch.tensor([0, rows // 3, rows])
    x, b = codes(g, 1, rows, m)[0], codes(g, groups, n, m)
    xs, bs = torch.rand(rows, 4, generator=g, device="cuda"), torch.rand(groups, -(-n // 128), 4, generator=g, device="cuda") / 1e4

    def run(x, xs, b, bs):
        Y = torch.empty(rows, n, dtype=TYPES[typ], device="cuda")
        nmf.nmf_grouped_product8(x, xs, cut.cuda(), groups, rows, b, bs, True, m, n, Y)
        return Y

    want = run(x, xs, b, bs)
    nan = torch.tensor(math.nan).to(E8).cuda()
    x2, xs2, b2 = x.clone(), xs.clone(), b.clone()
    x2.view(torch.uint8)[rows - 1, 5] = nan.view(torch.uint8)
    xs2[0, 3] = math.nan
    b2.view(torch.uint8)[1, 7, 399] = nan.view(torch.uint8)
    got = run(x2, xs2, b2, bs)
    bad = torch.zeros(rows, n, dtype=torch.bool, device="cuda")
    bad[rows - 1], bad[0] = True, True
    bad[rows // 3:, 7] = True
    assert bool(got[bad].isnan().all()) and torch.equal(got[~bad], want[~bad])


# ---- routing -----------------------------------------------------------------------------------

def route(logits, k, normalise, work=None, stream=None):
    rows, groups = logits.shape
    choice, place = (torch.full((rows, k), 77, dtype=torch.int32, device="cuda") for _ in range(2))
    gate, balance = torch.full((rows, k), 77.0, device="cuda"), torch.full((1,), 77.0, device="cuda")
    offsets = torch.full((groups + 1,), 77, dtype=torch.int64, device="cuda")
    nmf.nmf_route(logits, rows, groups, k, normalise, choice, gate, offsets, place, balance, work=work, stream=stream)
    return choice, gate, offsets, place, balance


def by_definition(logits, k, normalise):
    """Everything from the logits in 64 bits, on the host."""
    l = logits.double().cpu()
    rows, groups = l.shape
    order = torch.where(l.isnan(), -math.inf, l)
    top, at = torch.sort(order, dim=1, descending=True, stable=True)
    chosen = top[:, :k] > -math.inf
    choice = torch.where(chosen, at[:, :k], -1)
    alive = chosen.any(1)
    p = torch.zeros_like(l)
    p[alive] = torch.softmax(l[alive], dim=1)
    gate = torch.where(chosen, p.gather(1, choice.clamp_min(0)), 0.0)
    if normalise:
        gate[alive] = gate[alive] / gate[alive].sum(1, keepdim=True)
    flat = torch.where(chosen, choice, groups).reshape(-1)
    counts = torch.bincount(flat, minlength=groups + 1)[:groups]
    offsets = torch.cat([torch.zeros(1, dtype=torch.int64), counts.cumsum(0)])
    order = torch.argsort(flat, stable=True)
    place = torch.empty_like(order)
    place[order] = torch.arange(rows * k)
    place = torch.where(chosen, place.view(rows, k), -1)
    C, mine = max(1, int(counts.sum())), chosen.sum(1, keepdim=True).double()
    parts = groups * counts.double() / C * (mine * p / C)
    return choice, gate, offsets, place, parts[alive].sum(), p, chosen, alive


def logits_of(kind, rows, groups, dt, g):
    l = 2 * normal(g, rows, groups) + normal(g, 1, groups)
    if kind == "ties":
        l = (l * 2).round() / 2
        l[::3] = 0.0
        l[::5] = -0.0
        l[::3, ::2] = -0.0
    elif kind == "masked":
        l[torch.rand(rows, groups, generator=g, device="cuda") < 0.6] = -math.inf
        l[rows // 2::4] = -math.inf
    elif kind == "lowest":
        l = l.to(dt)
        l[torch.rand(rows, groups, generator=g, device="cuda") < 0.7] = torch.finfo(dt).min
        l[::2] = torch.finfo(dt).min
    elif kind == "far":
        l = l * (300 if dt != torch.float16 else 1000)
    return l.to(dt)


ROUTES = [(1, 1, 1), (1, 2, 2), (3, 8, 2), (64, 8, 8), (65, 33, 16), (24, 64, 4), (300, 64, 6), (129, 100, 1), (1000, 128, 8), (77, 256, 16),
          (130, 257, 3), (200, 512, 8), (70, 1000, 16), (65, 1024, 4), (5000, 16, 2)]


@gpu
@pytest.mark.parametrize("typ", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("kind", ["plain", "ties", "masked", "lowest", "far"])
@pytest.mark.parametrize("rows,groups,k", ROUTES)
def test_route_and_its_gradient(rows, groups, k, kind, typ):
    dt = TYPES[typ]
    g = torch.Generator(device="cuda").manual_seed(rows + groups)
    pad = rows % 3
    logits = torch.full((rows, groups + pad), math.nan, dtype=dt, device="cuda")[:, :groups]
    logits.copy_(logits_of(kind, rows, groups, dt, g))
    for normalise in (False, True):
        got = [t.cpu() for t in route(logits, k, normalise)]
        want = by_definition(logits, k, normalise)
        for i in (0, 2, 3):
            assert torch.equal(got[i].long(), want[i]), i
        # exp of logits below the largest by more than 128 is nothing; what else is lost is in every p
        lost = (groups + 300) * U
        off = (got[1].double() - want[1]).abs()
        assert bool((off <= (2 * lost + k * U) * want[1] + 2.0 ** -126).all())
        assert abs(float(got[4]) - float(want[4])) <= (lost + (rows + groups) * U) * abs(float(want[4])) + 2.0 ** -126
        for other in (0, 1 << 20):                           # without scratch one workgroup does the same
            again = [t.cpu() for t in route(logits, k, normalise, work=torch.empty(other, dtype=torch.uint8, device="cuda"))]
            for i in range(4):
                assert torch.equal(again[i], got[i]), i
            assert abs(float(again[4]) - float(want[4])) <= (lost + (rows + groups) * U) * abs(float(want[4])) + 2.0 ** -126

        choice, gate, offsets, place, balance, p, chosen, alive = want
        dgate, db = normal(g, rows, k), torch.tensor([0.7 * rows], device="cuda")
        dgate[~chosen.cuda()] = math.nan                     # not used
        C, counts, mine = max(1, int(offsets[-1])), offsets.diff().double(), chosen.sum(1, keepdim=True).double()
        for dg, dbal in ((dgate, db), (dgate, None), (None, db)):
            mem = torch.full((rows, groups + pad), 77.0, dtype=dt, device="cuda")
            nmf.nmf_route_gradient(logits, rows, groups, k, normalise, got[0].cuda(), got[2].cuda(), dg, dbal, mem[:, :groups])
            torch.cuda.synchronize()
            assert bool((mem[:, groups:] == torch.tensor(77.0).to(dt).item()).all())
            d, size = torch.zeros_like(p), torch.zeros_like(p)
            if dg is not None:
                w = torch.where(chosen, dg.cpu().double(), 0.0)
                at = choice.clamp_min(0)
                mean, big = (w * gate).sum(1, keepdim=True), (w.abs() * gate).sum(1, keepdim=True)
                if normalise:
                    d.scatter_add_(1, at, gate * (w - mean))
                    size.scatter_add_(1, at, gate * (w.abs() + big))
                else:
                    d.scatter_add_(1, at, gate * w)
                    size.scatter_add_(1, at, gate * w.abs())
                    d, size = d - p * mean, size + p * big
            if dbal is not None:
                q = float(dbal) * groups * counts / C ** 2
                d = d + mine * p * (q - (p * q).sum(1, keepdim=True))
                size = size + mine * p * (q + (p * q).sum(1, keepdim=True))
            near(mem[:, :groups].cpu(), d, typ, (4 * lost + 3 * k * U) * size + 2.0 ** -126)
            assert not bool(mem[:, :groups].cpu()[~alive].any())


@gpu
def test_route_gradient_against_differences():
    """Of sum(dgate gate) + dbalance balance, in one direction that changes no choice."""
    g = torch.Generator(device="cuda").manual_seed(21)
    rows, groups, k = 200, 12, 3
    l = torch.stack([torch.randperm(groups, generator=g, device="cuda") for _ in range(rows)]).float() * 0.25      # steps of 1 / 4 apart
    D = (2 * torch.rand(rows, groups, generator=g, device="cuda") - 1)
    dgate, db, step = normal(g, rows, k), torch.tensor([30.0], device="cuda"), 2.0 ** -6
    for normalise in (False, True):
        def loss(x):
            c, gate, _, _, b = route(x, k, normalise)
            return float((dgate.double() * gate.double()).sum() + 30.0 * b.double()), c
        base, choice = loss(l)
        values = []
        for s in (1, -1, 2, -2):
            v, c = loss(l + s * step * D)
            assert torch.equal(c, choice)
            values.append(v)
        four = (8 * (values[0] - values[1]) - (values[2] - values[3])) / (12 * step)
        offsets = route(l, k, normalise)[2]
        d = torch.empty_like(l)
        nmf.nmf_route_gradient(l, rows, groups, k, normalise, choice, offsets, dgate, db, d)
        # the losses are known to about 600 terms of 2^-22, over the step; the fifth derivative times step^4 is below that
        assert abs(four - float((d.double() * D.double()).sum())) < 600 * 2.0 ** -22 / step * 2


@gpu
@pytest.mark.parametrize("groups", [8, 100, 300])
@pytest.mark.parametrize("rows", [40, 200])
def test_route_of_what_is_not_finite(rows, groups):
    g = torch.Generator(device="cuda").manual_seed(22)
    k = 4
    l = normal(g, rows, groups)
    want = route(l, k, True)
    bad = l.clone()
    bad[3, 1], bad[9, 5], bad[11] = math.nan, math.inf, math.nan
    bad[13] = -math.inf
    bad[13, :2] = torch.tensor([math.nan, 0.5])
    got = route(bad, k, True)
    ref = by_definition(bad, k, True)
    for i in (0, 2, 3):
        assert torch.equal(got[i].cpu().long(), ref[i])
    ok = torch.ones(rows, dtype=torch.bool, device="cuda")
    ok[[3, 9, 11, 13]] = False
    assert torch.equal(got[0][ok], want[0][ok]) and torch.equal(got[1][ok], want[1][ok])
    assert bool(got[1][3].isnan().all()) and bool(got[1][9].isnan().all()) and int(got[0][9, 0]) == 5
    assert bool((got[0][11] == -1).all()) and bool((got[1][11] == 0).all())
    assert got[0][13].tolist() == [1, -1, -1, -1] and bool(got[1][13, 0].isnan()) and bool((got[1][13, 1:] == 0).all())
    assert bool(got[4].isnan())
    d, e = torch.empty_like(l), torch.empty_like(l)
    dg = normal(g, rows, k)
    db = torch.ones(1, device="cuda")
    nmf.nmf_route_gradient(bad, rows, groups, k, True, got[0], got[2], dg, None, d)
    nmf.nmf_route_gradient(l, rows, groups, k, True, want[0], want[2], dg, None, e)
    assert torch.equal(d[ok], e[ok]) and bool((d[11] == 0).all()) and bool(d[3].isnan().any())
    nmf.nmf_route_gradient(bad, rows, groups, k, True, got[0], got[2], dg, db, d)
    assert bool(d[ok].isfinite().all())
    # choices and offsets that are no such thing
    wild = torch.randint(-2 ** 31, 2 ** 31 - 1, (rows, k), generator=g, device="cuda").int()
    nmf.nmf_route_gradient(l, rows, groups, k, True, wild, torch.randint(-2 ** 62, 2 ** 62, (groups + 1,), generator=g, device="cuda"), dg, db, d)
    torch.cuda.synchronize()


@gpu
def test_route_of_no_rows_and_of_masked_rows_alone():
    for rows in (0, 5, 100):
        l = torch.full((rows, 6), -math.inf, device="cuda")
        choice, gate, offsets, place, balance = route(l, 2, True)
        assert not bool(offsets.any()) and float(balance) == 0 and bool((choice == -1).all()) and bool((place == -1).all()) and bool((gate == 0).all())
        if rows:
            d = torch.full_like(l, 5.0)
            nmf.nmf_route_gradient(l, rows, 6, 2, True, choice, offsets, torch.ones(rows, 2, device="cuda"), torch.ones(1, device="cuda"), d)
            assert not bool(d.any())


@gpu
def test_balance_is_one_where_all_groups_are_equal():
    groups, k = 16, 2
    l = torch.zeros(groups * 8, groups, device="cuda")
    at = torch.arange(groups * 8, device="cuda")
    l[at, at % groups] = 1e-3
    l[at, (at + 1) % groups] = 1e-3
    assert abs(float(route(l, k, False)[4]) - 1) < 1e-5
    l = torch.zeros(64, groups, device="cuda")
    l[:, 0] = 50.0                                            # all rows to the first group
    assert abs(float(route(l, 1, False)[4]) - groups) < 1e-4


@gpu
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("what", ["widths", "x", "b", "one"])
def test_product8_copies_rows_that_are_not_whole(what, transposed):
    """Long products of rows that do not begin or end on 16 bytes, with the scratch that copies take, with less, and with none."""
    g = torch.Generator(device="cuda").manual_seed(14)
    rows, groups, m, n = 3000, 2, 1500 if what in ("widths", "one") else 1504, 1501 if what in ("widths", "one") else 1504
    cut = torch.tensor([3, 1700, 2990])
    inside = (torch.arange(rows, device="cuda") >= 3) & (torch.arange(rows, device="cuda") < 2990)
    shape = (n, m) if transposed else (m, n)
    x, b = codes(g, 1, rows, m), codes(g, 1 if what == "one" else groups, *shape)
    xs, bs = torch.rand(rows, 12, generator=g, device="cuda"), torch.rand(b.shape[0], 12, 12, generator=g, device="cuda") / 1e4
    X, B = strided(x, 1 if what == "x" else 0, 0)[0], strided(b, 0, 5 if what == "b" else 0)
    if what == "one":
        B, bs = B.expand(groups, *shape), bs.expand(groups, 12, 12)
    want, size = product(x[0], xs, b.expand(groups, *shape), bs, cut, transposed)
    need = nmf.nmf_routed_work_bytes(2 | {"x": nmf.NMF_ODD_X, "b": nmf.NMF_ODD_B, "one": nmf.NMF_ONE_B, "widths": 0}[what], rows, m, n, groups)
    assert need >= rows * m if what == "x" else need >= m * n
    for work in (None, need, need - 16, 0):
        Y = torch.full((rows, n), 77.0, dtype=torch.bfloat16, device="cuda")
        nmf.nmf_grouped_product8(X, xs, cut.cuda(), groups, rows, B, bs, transposed, m, n, Y,
                                 work=None if work is None else torch.full((work,), 255, dtype=torch.uint8, device="cuda"))
        holds(Y, want, size, m, "bf16", inside)
        assert bool((Y[~inside] == 77).all())


@gpu
@pytest.mark.parametrize("rows,groups,k", [(16, 1024, 16), (17, 1024, 16), (32, 200, 5), (33, 200, 5), (64, 64, 8), (9000, 700, 4), (17000, 40, 2), (9000, 257, 1)])
def test_route_in_blocks_of_any_size(rows, groups, k):
    """Rows at the ends of what one workgroup takes, and so many that blocks have several turns."""
    g = torch.Generator(device="cuda").manual_seed(rows)
    l = (2 * normal(g, rows, groups)).to(torch.bfloat16)
    l[rows // 3:rows // 2] = -math.inf
    got = [t.cpu() for t in route(l, k, True)]
    want = by_definition(l, k, True)
    for i in (0, 2, 3):
        assert torch.equal(got[i].long(), want[i]), i
    lost = (groups + 300) * U
    assert bool(((got[1].double() - want[1]).abs() <= (2 * lost + k * U) * want[1] + 2.0 ** -126).all())
    assert abs(float(got[4]) - float(want[4])) <= (lost + (rows + groups) * U) * float(want[4])


@gpu
@pytest.mark.parametrize("n", [1, 5, 17, 63, 65, 129, 200])
@pytest.mark.parametrize("m", [127, 128, 129, 256, 300])
def test_product8_reads_nothing_behind_its_arrays(m, n):
    """Odd widths whose last rows end where the memory that may be read ends: codes behind it are NaN, and would show."""
    g = torch.Generator(device="cuda").manual_seed(m + n)
    for rows, typ in ((3, "bf16"), (90, "f32")):
        x, b = codes(g, 1, rows, m)[0], codes(g, 2, m, n)
        xs, bs = torch.rand(rows, -(-m // 128), generator=g, device="cuda"), torch.rand(2, -(-m // 128), -(-n // 128), generator=g, device="cuda") / 100
        cut = torch.tensor([0, rows // 2, rows])
        memx, memb = (torch.full((t.numel() + 4096,), 127, dtype=torch.uint8, device="cuda") for t in (x, b))
        X, B = memx[:x.numel()].view(rows, m), memb[:b.numel()].view(2, m, n)
        X.copy_(x.view(torch.uint8))
        B.copy_(b.view(torch.uint8))
        Y = torch.empty(rows, n, dtype=TYPES[typ], device="cuda")
        nmf.nmf_grouped_product8(X, xs, cut.cuda(), 2, rows, B, bs, False, m, n, Y)
        want, size = product(x, xs, b, bs, cut, False)
        holds(Y, want, size, m, typ, torch.ones(rows, dtype=torch.bool, device="cuda"))
        Bt = memb[:b.numel()].view(2, n, m)
        Bt.copy_(b.view(torch.uint8).transpose(1, 2))
        nmf.nmf_grouped_product8(X, xs, cut.cuda(), 2, rows, Bt, bs.transpose(1, 2).contiguous(), True, m, n, Y)
        holds(Y, want, size, m, typ, torch.ones(rows, dtype=torch.bool, device="cuda"))


@gpu
@pytest.mark.parametrize("transposed", [False, True])
def test_product8_of_long_contractions_in_large_tiles(transposed):
    """More than 64 blocks, whose scales come 64 at a time, the last one in part."""
    g = torch.Generator(device="cuda").manual_seed(15)
    rows, m, n = 2100, 8336, 4112
    M, N = -(-m // 128), -(-n // 128)
    x, b = codes(g, 1, rows, m)[0], codes(g, 1, *((n, m) if transposed else (m, n)))
    xs = torch.exp(normal(g, rows, M)) / 1000
    bs = torch.exp(normal(g, 1, *((N, M) if transposed else (M, N)))) / 60
    cut = torch.tensor([0, rows])
    want, size = product(x, xs, b, bs, cut, transposed)
    for typ in ("bf16", "f32"):
        Y = torch.empty(rows, n, dtype=TYPES[typ], device="cuda")
        nmf.nmf_grouped_product8(x, xs, cut.cuda(), 1, rows, b, bs, transposed, m, n, Y)
        holds(Y, want, size, m, typ, torch.ones(rows, dtype=torch.bool, device="cuda"))

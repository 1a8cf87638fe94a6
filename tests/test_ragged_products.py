"""Products over ragged ranges of rows against their definitions in 64 bits.

Bounds, entry by entry: an output in bf16 or f16 is off by half a unit of its last place (at most 2^-8 or 2^-11 of it; 2^-25
below f16's normal range) and by the sum's own error.  A sum of K products held in fp32 loses at most 2^-23 of the sum
of the magnitudes per addition, whatever the order and the rounding: K 2^-23 of it.  Factors that meet 16-bit types go as
two bf16 pieces: 2^-17 of the magnitudes.
"""
import ctypes

import numpy as np
import pytest
import torch

import paper_2202_09518_amd as nmf

gpu = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}


def within(got, want, size, terms, typ, extra=0.0):
    """got against want (64 bits); size: the same sums over magnitudes; extra: further absolute bound."""
    got = got.double()
    bound = HALF[typ] * want.abs() + terms * 2.0 ** -23 * size * (1 + HALF[typ]) + 2.0 ** -25 + extra
    off = (got - want).abs()
    bad = ~(off <= bound)
    assert not bool(bad.any()), (int(bad.sum()), float((off / bound).nan_to_num(1e30).max()))


def padded(rows, cols, dtype, g, pad, first):
    """A rows x cols view with leading dimension cols + pad that starts `first` entries into its memory, random; and the memory."""
    mem = torch.full(((rows + 1) * (cols + pad) + first,), float("nan"), dtype=dtype, device="cuda")
    view = mem.as_strided((rows, cols), (cols + pad, 1), first)
    view.copy_(torch.randn(rows, cols, generator=g, device="cuda"))
    return view, mem


def result(rows, cols, dtype, pad, first):
    mem = torch.full(((rows + 1) * (cols + pad) + first,), 77.0, dtype=dtype, device="cuda")
    return mem.as_strided((rows, cols), (cols + pad, 1), first), mem


def untouched(mem, view, pad, first, rows_written=None):
    """Nothing but the view was written."""
    keep = mem.clone()
    keep.as_strided(view.shape, view.stride(), first).fill_(77.0)
    assert bool((keep == 77.0).all())


def lengths_of(kind, rows, parts, seed):
    r = np.random.default_rng(seed)
    if kind == "even":
        cut = np.linspace(0, rows, parts + 1).astype(np.int64)
    elif kind == "one":                       # all rows in one range, empty ones around it
        cut = np.array([0] * (parts // 2 + 1) + [rows] * (parts - parts // 2), dtype=np.int64)
    else:
        cut = np.concatenate([[0], np.sort(r.integers(0, rows + 1, parts - 1)), [rows]]).astype(np.int64)
    return cut


# rows, groups, m, n, lengths: one row, one column, k below a stage, odd sizes, every tile shape, split contractions
GROUPED = [
    (1, 1, 1, 1, "even"), (1, 3, 64, 8, "one"), (5, 4, 7, 3, "ragged"), (33, 5, 130, 65, "ragged"),
    (40, 70, 96, 136, "ragged"), (24, 16, 2048, 256, "ragged"), (200, 3, 257, 129, "ragged"), (300, 2, 1000, 520, "ragged"),
    (130, 1, 4096, 264, "even"), (700, 9, 64, 384, "one"), (3400, 1, 200, 4100, "even"), (3400, 3, 72, 4096, "ragged"),
]


@gpu
@pytest.mark.parametrize("typ", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("rows,groups,m,n,kind", GROUPED)
def test_grouped_product(rows, groups, m, n, kind, transposed, typ):
    g = torch.Generator(device="cuda").manual_seed(rows + m)
    dt = TYPES[typ]
    cut = lengths_of(kind, rows, groups, rows)
    off = torch.from_numpy(cut).cuda()
    aligned = m % 8 == 0 and n % 8 == 0
    pad, first = (8, 16) if aligned else (1, 1)
    X, _ = padded(rows, m, dt, g, pad, first)
    B = torch.randn(groups, *((n, m) if transposed else (m, n)), generator=g, device="cuda").to(dt)
    Y, mem = result(rows, n, dt, pad, first)
    nmf.nmf_grouped_product(X, off, groups, rows, B, transposed, m, n, Y)
    torch.cuda.synchronize()
    untouched(mem, Y, pad, first)
    for i in range(groups):
        a, b = int(cut[i]), int(cut[i + 1])
        if a == b:
            continue
        x, w = X[a:b].double(), B[i].double()
        w = w.t().contiguous() if transposed else w
        within(Y[a:b], x @ w, x.abs() @ w.abs(), m, typ)
    # without scratch: the contraction in one piece
    Z, _ = result(rows, n, dt, pad, first)
    nmf.nmf_grouped_product(X, off, groups, rows, B, transposed, m, n, Z, work=torch.empty(0, dtype=torch.uint8, device="cuda"))
    for i in range(groups):
        a, b = int(cut[i]), int(cut[i + 1])
        x, w = X[a:b].double(), B[i].double()
        w = w.t().contiguous() if transposed else w
        within(Z[a:b], x @ w, x.abs() @ w.abs(), m, typ)


@gpu
@pytest.mark.parametrize("typ", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,groups,m,n,kind", [
    (1, 1, 1, 1, "even"), (1, 2, 9, 70, "one"), (63, 4, 130, 66, "ragged"), (500, 1, 136, 264, "even"), (2000, 3, 129, 257, "ragged"),
    (300, 64, 64, 72, "ragged"), (1500, 2, 264, 520, "one"), (100, 2, 3336, 2600, "ragged"),
])
def test_grouped_gradient(rows, groups, m, n, kind, typ):
    g = torch.Generator(device="cuda").manual_seed(rows + m)
    dt = TYPES[typ]
    cut = lengths_of(kind, rows, groups, rows)
    off = torch.from_numpy(cut).cuda()
    pad, first = (8, 16) if m % 8 == 0 and n % 8 == 0 else (3, 1)
    X, _ = padded(rows, m, dt, g, pad, first)
    dY, _ = padded(rows, n, dt, g, pad, first)
    mem = torch.full((groups * m * (n + 4) + 4,), 77.0, dtype=dt, device="cuda")
    G = mem.as_strided((groups, m, n), (m * (n + 4), n + 4, 1), 0)
    for work in (None, torch.empty(0, dtype=torch.uint8, device="cuda")):
        G.fill_(5.0)
        nmf.nmf_grouped_gradient(X, dY, off, groups, rows, m, n, G, work=work)
        torch.cuda.synchronize()
        untouched(mem, G, 4, 0)
        for i in range(groups):
            x, dy = X[cut[i]:cut[i + 1]].double(), dY[cut[i]:cut[i + 1]].double()
            within(G[i], x.t() @ dy, x.abs().t() @ dy.abs(), max(1, int(cut[i + 1] - cut[i])), typ)
            if cut[i] == cut[i + 1]:
                assert bool((G[i] == 0).all())


class Problem:
    """Adapters of segments of rows: inputs, and what the definitions give in 64 bits."""

    def __init__(self, rows, segments, runs, kmin, kmax, m, n, transposed, typ, kind="ragged", none=True, seed=1):
        r = np.random.default_rng(seed + rows)
        g = torch.Generator(device="cuda").manual_seed(seed + m)
        dt = TYPES[typ]
        self.__dict__.update(rows=rows, segments=segments, runs=runs, kmax=kmax, m=m, n=n, transposed=transposed, typ=typ)
        self.cut = lengths_of(kind, rows, segments, seed)
        self.which = r.integers(0, runs, segments)
        if none and segments > 2:
            self.which[segments // 2] = -1
        self.ranks = [kmin + (kmax - kmin) * i // max(1, runs - 1) for i in range(runs)]
        self.ko = np.cumsum([0] + self.ranks)
        self.ktotal = int(self.ko[-1])
        self.offsets = torch.from_numpy(self.cut).cuda()
        self.run = torch.tensor(self.which, dtype=torch.int32, device="cuda")
        self.koff = torch.tensor(self.ko, dtype=torch.int32, device="cuda")
        pad, first = (8, 16) if m % 8 == 0 and n % 8 == 0 else (1, 1)
        self.pad, self.first = pad, first
        self.X, _ = padded(rows, m, dt, g, pad, first)
        self.dY, _ = padded(rows, n, dt, g, pad, first)
        self.A, _ = padded(*((n, m) if transposed else (m, n)), dt, g, pad, first)
        self.Wt = (torch.randn(self.ktotal, m, generator=g, device="cuda") / m ** 0.5).to(dt)
        self.H = torch.randn(self.ktotal, n, generator=g, device="cuda").to(dt)
        self.scale = torch.rand(runs, generator=g, device="cuda") + 0.5
        self.U = torch.full((rows, kmax), float("nan"), device="cuda")
        self.V = torch.full((rows, kmax), float("nan"), device="cuda")

    def forward(self, Y, work=None, stream=None):
        p = self
        nmf.nmf_lowrank_product(p.X, p.rows, p.A, p.transposed, p.m, p.n, p.offsets, p.run, p.segments, p.Wt, p.H, p.koff, p.runs, p.kmax,
                                p.scale, p.U, Y, work=work, stream=stream)

    def backward(self, dX, dWt, dH, work=None):
        p = self
        nmf.nmf_lowrank_product(p.dY, p.rows, p.A, not p.transposed, p.n, p.m, p.offsets, p.run, p.segments, p.H, p.Wt, p.koff, p.runs,
                                p.kmax, p.scale, p.V, dX, work=work)
        nmf.nmf_lowrank_gradient(p.X, p.dY, p.rows, p.m, p.n, p.offsets, p.run, p.segments, p.koff, p.runs, p.kmax, p.U, p.V, dWt, dH,
                                 work=work)

    def parts(self):
        for i in range(self.segments):
            a, b, r = int(self.cut[i]), int(self.cut[i + 1]), int(self.which[i])
            if r >= 0 and b > a:
                yield slice(a, b), slice(int(self.ko[r]), int(self.ko[r + 1])), float(self.scale[r])

    def check_product(self, Y, X, A, down, up, U):
        """Y = X A + U up, U = scale X down^T; all 64 bits but Y and U."""
        Yw, size = X @ A, X.abs() @ A.abs()
        K = A.shape[0]
        low = torch.zeros_like(Yw)
        for rows, k, s in self.parts():
            u, us = X[rows] @ down[k].t() * s, X[rows].abs() @ down[k].abs().t() * s
            kr = k.stop - k.start
            assert not bool(torch.isnan(U[rows, :kr]).any())
            off = (U[rows, :kr].double() - u).abs()
            assert bool((off <= (K + 2) * 2.0 ** -23 * us).all())
            Yw[rows] += u @ up[k]
            size[rows] += us @ up[k].abs()
            low[rows] += u.abs() @ up[k].abs()
        pieces = 0.0 if self.typ == "f32" else 2.0 ** -17 * low
        within(Y, Yw, size, K + self.kmax + 2, self.typ, pieces)

    def check_gradient(self, dWt, dH):
        X, dY = self.X.double(), self.dY.double()
        W, H = self.Wt.double(), self.H.double()
        gw, gh = torch.zeros_like(W), torch.zeros_like(H)
        sw, sh = torch.zeros_like(W), torch.zeros_like(H)
        for rows, k, s in self.parts():
            v, u = dY[rows] @ H[k].t() * s, X[rows] @ W[k].t() * s
            gw[k] += v.t() @ X[rows]
            gh[k] += u.t() @ dY[rows]
            sw[k] += (dY[rows].abs() @ H[k].abs().t() * s).t() @ X[rows].abs()
            sh[k] += (X[rows].abs() @ W[k].abs().t() * s).t() @ dY[rows].abs()
        pieces = 0.0 if self.typ == "f32" else 2.0 ** -17
        within(dWt, gw, sw, self.rows + self.n + 2, self.typ, pieces * sw)
        within(dH, gh, sh, self.rows + self.m + 2, self.typ, pieces * sh)


# rows, segments, runs, kmin, kmax, m, n, lengths
LOWRANK = [
    (1, 1, 1, 1, 1, 1, 1, "even"), (1, 1, 8, 16, 16, 2048, 256, "even"), (48, 48, 15, 2, 16, 512, 320, "even"),
    (7, 5, 3, 1, 5, 33, 9, "ragged"), (160, 40, 24, 8, 64, 1024, 264, "ragged"), (300, 70, 7, 3, 33, 130, 257, "ragged"),
    (129, 4, 2, 100, 256, 200, 136, "ragged"), (3400, 6, 4, 8, 40, 128, 4100, "ragged"), (3400, 9, 3, 64, 70, 136, 4096, "one"),
    (1000, 3, 2, 4, 4, 72, 72, "even"),
]


@gpu
@pytest.mark.parametrize("typ", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("rows,segments,runs,kmin,kmax,m,n,kind", LOWRANK)
def test_lowrank_forward_and_backward(rows, segments, runs, kmin, kmax, m, n, kind, transposed, typ):
    p = Problem(rows, segments, runs, kmin, kmax, m, n, transposed, typ, kind)
    X, dY, A = p.X.double(), p.dY.double(), p.A.double()
    A = A.t().contiguous() if transposed else A
    W, H = p.Wt.double(), p.H.double()
    for work in (None, torch.empty(0, dtype=torch.uint8, device="cuda")):
        p.U.fill_(float("nan"))
        p.V.fill_(float("nan"))
        Y, ymem = result(rows, n, TYPES[typ], p.pad, p.first)
        dX, xmem = result(rows, m, TYPES[typ], p.pad, p.first)
        dWt, dH = torch.full_like(p.Wt, 5.0), torch.full_like(p.H, 5.0)
        p.forward(Y, work)
        p.backward(dX, dWt, dH, work)
        torch.cuda.synchronize()
        untouched(ymem, Y, p.pad, p.first)
        untouched(xmem, dX, p.pad, p.first)
        p.check_product(Y, X, A, W, H, p.U)
        p.check_product(dX, dY, A.t().contiguous(), H, W, p.V)
        p.check_gradient(dWt, dH)


@gpu
@pytest.mark.parametrize("rows,segments,m,n", [(40, 5, 200, 136), (600, 4, 65, 130)])
def test_factor_gradients_against_differences(rows, segments, m, n):
    """<Y, dY> is linear in W and in H: half of its difference over +D and -D is the gradient's product with D, up to the
    roundings of Y (2^-24 of each entry, and (K + k) 2^-23 of the magnitudes in its sum) on either side."""
    p = Problem(rows, segments, 3, 4, 12, m, n, False, "f32")
    Y, dX = torch.empty(rows, n, device="cuda"), torch.empty(rows, m, device="cuda")
    dWt, dH = torch.empty_like(p.Wt), torch.empty_like(p.H)
    p.forward(Y)
    p.backward(dX, dWt, dH)
    for name, grad in (("Wt", dWt), ("H", dH)):
        base = getattr(p, name).clone()
        D = torch.randn_like(base)
        value, size = [], 0.0
        for sign in (1.0, -1.0):
            setattr(p, name, (base + sign * D).contiguous())
            p.forward(Y)
            value.append(float((Y.double() * p.dY.double()).sum()))
            mag = p.X.double().abs() @ p.A.double().abs()
            for r, k, s in p.parts():
                mag[r] += p.X[r].double().abs() @ p.Wt[k].double().abs().t() * s @ p.H[k].double().abs()
            size += float((mag * p.dY.double().abs()).sum())
        setattr(p, name, base)
        want = (value[0] - value[1]) / 2
        have = float((grad.double() * D.double()).sum())
        # base +- D is itself rounded: 2^-24 of the factors, which the same sum of magnitudes bounds
        assert abs(want - have) <= (m + n + rows + 16) * 2.0 ** -23 * size


@gpu
@pytest.mark.parametrize("typ", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,m,n", [(48, 256, 200), (700, 96, 136), (3400, 72, 4096)])
def test_what_is_not_finite_stays_in_its_rows(rows, m, n, typ):
    p = Problem(rows, 6, 6, 4, 9, m, n, True, typ, none=False)
    p.which = np.arange(6)
    p.run = torch.arange(6, dtype=torch.int32, device="cuda")
    Y, Z = (torch.empty(rows, n, dtype=TYPES[typ], device="cuda") for _ in range(2))
    p.forward(Y)
    p.X[int(p.cut[1])] = float("inf")                 # one row; and the factors of another run
    p.H[p.ko[3]:p.ko[4]] = float("nan")
    p.Wt[p.ko[4]:p.ko[5]] = float("inf")
    p.forward(Z)
    torch.cuda.synchronize()
    clean = torch.ones(rows, dtype=torch.bool, device="cuda")
    if p.cut[2] > p.cut[1]:
        clean[int(p.cut[1])] = False
    for s in (3, 4):
        clean[int(p.cut[s]):int(p.cut[s + 1])] = False
        assert not bool(torch.isfinite(Z[int(p.cut[s]):int(p.cut[s + 1])].float()).any())
    assert torch.equal(Y[clean], Z[clean])
    # groups
    off = p.offsets
    B = torch.randn(6, m, n, device="cuda").to(TYPES[typ])
    X = torch.randn(rows, m, device="cuda").to(TYPES[typ])
    nmf.nmf_grouped_product(X, off, 6, rows, B, False, m, n, Y)
    B[2] = float("nan")
    nmf.nmf_grouped_product(X, off, 6, rows, B, False, m, n, Z)
    clean[:] = True
    clean[int(p.cut[2]):int(p.cut[3])] = False
    assert torch.equal(Y[clean], Z[clean])
    G, F = (torch.empty(6, m, n, dtype=TYPES[typ], device="cuda") for _ in range(2))
    dY = torch.randn(rows, n, device="cuda").to(TYPES[typ])
    nmf.nmf_grouped_gradient(X, dY, off, 6, rows, m, n, G)
    X[int(p.cut[2]):int(p.cut[3])] = float("inf")
    nmf.nmf_grouped_gradient(X, dY, off, 6, rows, m, n, F)
    for i in (0, 1, 3, 4, 5):
        assert torch.equal(G[i], F[i])


@gpu
def test_infinite_products_are_infinite():
    """An infinity in a factor gives infinities, not NaN, where the formula does."""
    for typ in ("f32", "bf16", "f16"):
        p = Problem(20, 1, 1, 4, 4, 64, 64, True, typ, "even", none=False)
        p.X.fill_(1.0)
        p.Wt.fill_(1.0)
        p.H.fill_(1.0)
        p.H[1, 5] = float("inf")
        Y = torch.empty(20, 64, dtype=TYPES[typ], device="cuda")
        p.forward(Y)
        assert bool((Y[:, 5] == float("inf")).all()) and bool(torch.isfinite(Y[:, :5].float()).all())


@gpu
def test_rows_outside_all_ranges():
    X = torch.randn(50, 64, device="cuda")
    B = torch.randn(2, 64, 32, device="cuda")
    Y = torch.full((50, 32), 9.0, device="cuda")
    nmf.nmf_grouped_product(X, torch.tensor([10, 20, 30], device="cuda"), 2, 50, B, False, 64, 32, Y)
    assert bool((Y[:10] == 9).all()) and bool((Y[30:] == 9).all()) and not bool((Y[10:30] == 9).any())


@gpu
def test_malformed_ranges_touch_nothing_outside():
    rows = 100
    X = torch.randn(rows, 64, device="cuda")
    B = torch.randn(4, 64, 32, device="cuda")
    mem = torch.full((rows + 64, 32), 7.0, device="cuda")
    Y = mem[32:32 + rows]
    off = torch.tensor([-5, 1 << 40, 3, 90, 1000], device="cuda")
    nmf.nmf_grouped_product(X, off, 4, rows, B, False, 64, 32, Y)
    G = torch.empty(4, 64, 32, device="cuda")
    nmf.nmf_grouped_gradient(X, Y, off, 4, rows, 64, 32, G)
    U = torch.empty(rows, 8, device="cuda")
    run = torch.tensor([7, -3, 0, 1], dtype=torch.int32, device="cuda")
    koff = torch.tensor([-4, 500, 6], dtype=torch.int32, device="cuda")
    Wt, H = torch.randn(12, 64, device="cuda"), torch.randn(12, 32, device="cuda")
    nmf.nmf_lowrank_product(X, rows, B[0], False, 64, 32, off, run, 4, Wt, H, koff, 2, 8, None, U, Y)
    nmf.nmf_lowrank_gradient(X, Y, rows, 64, 32, off, run, 4, koff, 2, 8, U, U, torch.empty_like(Wt), torch.empty_like(H))
    torch.cuda.synchronize()
    assert bool((mem[:32] == 7).all()) and bool((mem[32 + rows:] == 7).all())


@gpu
def test_one_matrix_for_all_groups_and_no_scale():
    X = torch.randn(90, 72, device="cuda")
    B = torch.randn(1, 72, 40, device="cuda")
    off = torch.tensor([0, 20, 21, 90], device="cuda")
    Y = torch.empty(90, 40, device="cuda")
    nmf.nmf_grouped_product(X, off, 3, 90, B.expand(3, 72, 40), False, 72, 40, Y)
    x, b = X.double(), B[0].double()
    within(Y, x @ b, x.abs() @ b.abs(), 72, "f32")
    p = Problem(90, 3, 2, 3, 5, 72, 40, False, "f32", none=False)
    Z = torch.empty(90, 40, device="cuda")
    p.scale.fill_(1.0)
    p.forward(Y)
    nmf.nmf_lowrank_product(p.X, 90, p.A, False, 72, 40, p.offsets, p.run, 3, p.Wt, p.H, p.koff, 2, 5, None, p.U, Z)
    assert torch.equal(Y, Z)


@gpu
def test_no_segments_and_no_rows():
    A = torch.randn(64, 48, device="cuda")
    X = torch.randn(10, 64, device="cuda")
    Y = torch.empty(10, 48, device="cuda")
    e32, e64 = torch.empty(0, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    Wt, H, koff = torch.randn(3, 64, device="cuda"), torch.randn(3, 48, device="cuda"), torch.tensor([0, 3], dtype=torch.int32, device="cuda")
    nmf.nmf_lowrank_product(X, 10, A, False, 64, 48, e64, e32, 0, Wt, H, koff, 1, 3, None, torch.empty(10, 3, device="cuda"), Y)
    within(Y, X.double() @ A.double(), X.double().abs() @ A.double().abs(), 64, "f32")
    G = torch.full((2, 64, 48), 5.0, device="cuda")
    off = torch.zeros(3, dtype=torch.int64, device="cuda")
    nmf.nmf_grouped_gradient(X[:0], Y[:0], off, 2, 0, 64, 48, G)
    assert bool((G == 0).all())
    nmf.nmf_grouped_product(X[:0], off, 2, 0, torch.randn(2, 64, 48, device="cuda"), False, 64, 48, Y[:0])
    dW, dH = torch.full_like(Wt, 5.0), torch.full_like(H, 5.0)
    U = torch.empty(0, 3, device="cuda")
    nmf.nmf_lowrank_gradient(X[:0], Y[:0], 0, 64, 48, e64, e32, 0, koff, 1, 3, U, U, dW, dH)
    assert bool((dW == 0).all()) and bool((dH == 0).all())


@gpu
def test_results_repeat_bit_for_bit_and_on_other_streams():
    p = Problem(500, 20, 5, 4, 40, 520, 264, False, "bf16")
    outs = []
    side = torch.cuda.Stream()
    for s in (None, side, None, side):
        Y = torch.empty(500, 264, dtype=torch.bfloat16, device="cuda")
        dX, dWt, dH = torch.empty(500, 520, dtype=torch.bfloat16, device="cuda"), torch.empty_like(p.Wt), torch.empty_like(p.H)
        torch.cuda.synchronize()
        if s is None:
            p.forward(Y)
            p.backward(dX, dWt, dH)
        else:
            with torch.cuda.stream(s):
                p.forward(Y)
                p.backward(dX, dWt, dH)
        torch.cuda.synchronize()
        outs.append((Y, dX, dWt, dH))
    for o in outs[1:]:
        for a, b in zip(o, outs[0]):
            assert torch.equal(a, b)
    Y = torch.empty(500, 264, dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    p.forward(Y, stream=side)                # a stream that is not the current one
    side.synchronize()
    assert torch.equal(Y, outs[0][0])


@gpu
def test_calls_are_captured():
    p = Problem(40, 10, 4, 4, 16, 1024, 264, True, "bf16")
    Y = torch.empty(40, 264, dtype=torch.bfloat16, device="cuda")
    dX, dWt, dH = torch.empty(40, 1024, dtype=torch.bfloat16, device="cuda"), torch.empty_like(p.Wt), torch.empty_like(p.H)
    p.forward(Y)
    p.backward(dX, dWt, dH)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.forward(Y)
        p.backward(dX, dWt, dH)
    for i in range(3):
        p.X.copy_(torch.randn(40, 1024, device="cuda"))
        for t in (Y, dX, dWt, dH):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (Y, dX, dWt, dH)]
        p.forward(Y)
        p.backward(dX, dWt, dH)
        torch.cuda.synchronize()
        for a, b in zip(got, (Y, dX, dWt, dH)):
            assert torch.equal(a, b)
    del graph


@gpu
def test_offsets_beyond_32_bits():
    """Entries more than 2^31 (and bytes more than 2^32) from the first: long rows far apart, and the last group of many."""
    rows, m, n = 70, 64, 64
    ld = 40_000_000                                       # 70 rows: 2.8e9 entries of 2 bytes
    mem = torch.empty(rows * ld, dtype=torch.bfloat16, device="cuda")
    X = mem.as_strided((rows, m), (ld, 1), 0)
    X.copy_(torch.randn(rows, m, device="cuda"))
    groups = 3
    stride = 1_200_000_000
    B = mem.as_strided((groups, m, n), (stride, n, 1), 128)
    B.copy_(torch.randn(groups, m, n, device="cuda"))
    X.copy_(torch.randn(rows, m, device="cuda"))
    Y = torch.empty(rows, n, dtype=torch.bfloat16, device="cuda")
    cut = [0, 3, 10, 70]
    off = torch.tensor(cut, device="cuda")
    nmf.nmf_grouped_product(X, off, groups, rows, B, False, m, n, Y)
    G = torch.empty(groups, m, n, dtype=torch.bfloat16, device="cuda")
    nmf.nmf_grouped_gradient(X, Y, off, groups, rows, m, n, G)
    for i in range(groups):
        x, b = X[cut[i]:cut[i + 1]].double(), B[i].double()
        within(Y[cut[i]:cut[i + 1]], x @ b, x.abs() @ b.abs(), m, "bf16")
        y = Y[cut[i]:cut[i + 1]].double()
        within(G[i], x.t() @ y, x.abs().t() @ y.abs(), rows, "bf16")


def test_ragged_arguments_are_refused():
    """Argument checks come before any call of the device."""
    L = nmf.lib()
    one, odd, null = ctypes.c_void_p(256), ctypes.c_void_p(257), ctypes.c_void_p(0)
    bad = nmf.NMF_EINVAL

    def product(type=1, X=one, ldx=8, off=one, groups=2, rows=4, B=one, ldb=8, stride=64, t=0, m=8, n=8, Y=one, ldy=8, work=null, wb=0):
        return L.nmf_grouped_product(type, X, ldx, off, groups, rows, B, ldb, stride, t, m, n, Y, ldy, work, wb, null)

    for kw in (dict(type=3), dict(type=-1), dict(X=null), dict(off=null), dict(B=null), dict(Y=null), dict(X=odd), dict(B=odd), dict(Y=odd),
               dict(off=odd), dict(ldx=7), dict(ldy=7), dict(ldb=7), dict(stride=-1), dict(groups=0), dict(rows=-1), dict(m=0), dict(n=0),
               dict(m=1 << 31), dict(wb=16), dict(work=odd, wb=16)):
        assert product(**kw) == bad, kw
        assert nmf.nmf_last_error() != ""
    assert product(rows=0) == nmf.NMF_OK
    assert product(rows=(1 << 31) - 1, n=(1 << 31) - 1, ldb=1 << 31, ldy=1 << 31) == nmf.NMF_EUNSUPPORTED

    def gradient(type=2, X=one, ldx=8, dY=one, ldy=8, off=one, groups=2, rows=4, m=8, n=8, G=one, ldg=8, stride=64, work=null, wb=0):
        return L.nmf_grouped_gradient(type, X, ldx, dY, ldy, off, groups, rows, m, n, G, ldg, stride, work, wb, null)

    for kw in (dict(type=9), dict(X=null), dict(dY=null), dict(off=null), dict(G=null), dict(ldx=7), dict(ldy=7), dict(ldg=7), dict(stride=63),
               dict(groups=0), dict(rows=-1), dict(m=0), dict(n=-1), dict(wb=1)):
        assert gradient(**kw) == bad, kw

    def lowrank(type=0, X=one, ldx=8, rows=4, A=one, lda=8, t=0, m=8, n=8, off=one, run=one, seg=2, Wt=one, H=one, koff=one, runs=2, kmax=4,
                ktotal=8, scale=null, U=one, Y=one, ldy=8, work=null, wb=0):
        return L.nmf_lowrank_product(type, X, ldx, rows, A, lda, t, m, n, off, run, seg, Wt, H, koff, runs, kmax, ktotal, scale, U, Y, ldy,
                                     work, wb, null)

    for kw in (dict(type=4), dict(X=null), dict(A=null), dict(Y=null), dict(off=null), dict(run=null), dict(Wt=null), dict(H=null),
               dict(koff=null), dict(U=null), dict(X=odd), dict(U=odd), dict(scale=odd), dict(ldx=7), dict(lda=7), dict(ldy=7), dict(seg=-1),
               dict(runs=0), dict(kmax=0), dict(ktotal=0), dict(rows=-2), dict(wb=8)):
        assert lowrank(**kw) == bad, kw
    assert lowrank(kmax=257) == nmf.NMF_EUNSUPPORTED
    assert lowrank(rows=0) == nmf.NMF_OK

    def factors(type=0, X=one, ldx=8, dY=one, ldy=8, rows=4, m=8, n=8, off=one, run=one, seg=2, koff=one, runs=2, kmax=4, ktotal=8, U=one,
                V=one, dW=one, dH=one, work=null, wb=0):
        return L.nmf_lowrank_gradient(type, X, ldx, dY, ldy, rows, m, n, off, run, seg, koff, runs, kmax, ktotal, U, V, dW, dH, work, wb, null)

    for kw in (dict(type=4), dict(X=null), dict(dY=null), dict(off=null), dict(run=null), dict(koff=null), dict(U=null), dict(V=null),
               dict(dW=null), dict(dH=null), dict(ldx=7), dict(ldy=7), dict(seg=-1), dict(runs=0), dict(kmax=0), dict(ktotal=0), dict(V=odd)):
        assert factors(**kw) == bad, kw
    assert factors(kmax=300) == nmf.NMF_EUNSUPPORTED


def test_ragged_work_bytes():
    wb = nmf.nmf_ragged_work_bytes
    assert wb(0, 3, 10, 64, 64, 1) == 0 and wb(9, 1, 10, 64, 64, 1) == 0 and wb(0, 1, 0, 64, 64, 1) == 0
    assert wb(0, 1, 16384, 4096, 4096, 1) == 0                       # tiles enough
    one = wb(0, 1, 16, 4096, 256, 1)                                 # few tiles: whole parts of the result
    assert one > 0 and one % (16 * 256 * 4) == 0
    assert wb(2, 1, 16, 4096, 256, 4, 2, 16, 32) > one               # and parts of U


def test_tensors_that_do_not_fit_are_refused():
    X = torch.zeros(4, 8)
    off = torch.zeros(3, dtype=torch.int64)
    with pytest.raises(ValueError):
        nmf.nmf_grouped_product(X, off, 2, 4, torch.zeros(2, 8, 8), False, 8, 8, torch.zeros(4, 8))
    with pytest.raises(ValueError):
        nmf.nmf_lowrank_gradient(X, X, 4, 8, 8, off, off, 2, off, 2, 4, X, X, X, X)


@gpu
def test_shapes_that_do_not_match_are_refused():
    X = torch.zeros(4, 8, device="cuda")
    off = torch.zeros(3, dtype=torch.int64, device="cuda")
    B, Y = torch.zeros(2, 8, 8, device="cuda"), torch.zeros(4, 8, device="cuda")
    call = nmf.nmf_grouped_product
    for args in ((X.half(), off, 2, 4, B, False, 8, 8, Y), (X, off[:2], 2, 4, B, False, 8, 8, Y), (X, off.int(), 2, 4, B, False, 8, 8, Y),
                 (X, off, 2, 4, B[:1], False, 8, 8, Y), (X, off, 2, 4, B, False, 8, 8, Y[:3]), (X, off, 2, 5, B, False, 8, 8, Y),
                 (X, off, 2, 4, B.transpose(1, 2), False, 8, 8, Y), (X.double(), off, 2, 4, B, False, 8, 8, Y)):
        with pytest.raises(ValueError):
            call(*args)

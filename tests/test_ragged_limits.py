"""What the products over ragged ranges keep to: their scratch on malformed offsets, its size, and the parts that it holds."""
import pytest
import torch

import paper_2202_09518_amd as nmf
from test_ragged_products import TYPES, Problem, lengths_of, within

gpu = pytest.mark.gpu


def overlapping(rows, segments):
    """Offsets that go back and forth: every second segment has all rows."""
    return [rows * (i % 2) for i in range(segments + 1)]


OVERLAP = dict(rows=4096, segments=64, m=128, n=136, kmax=16)


def chunks_planned(typ, block):
    """Chunks that the scratch has room for, and those that the rows of overlapping segments would fill at the planned length of
    four blocks each (the least)."""
    c = OVERLAP
    line = 32 * (c["m"] + c["n"]) * 4                               # one factor tile of 32, columns of both gradients
    pieces = 0 if typ == nmf.NMF_F32 else c["rows"] * 2 * 3 * 32 * 2
    room = (nmf.nmf_ragged_work_bytes(3, typ, c["rows"], c["m"], c["n"], c["segments"], 1, c["kmax"], c["kmax"]) - pieces) // line
    return room, c["segments"] // 2 * (c["rows"] // block) // 4


@pytest.mark.parametrize("typ,block", [(nmf.NMF_F32, 32), (nmf.NMF_BF16, 64), (nmf.NMF_F16, 32)])
def test_overlapping_segments_would_fill_more_chunks_than_there_are(typ, block):
    room, filled = chunks_planned(typ, block)
    assert 1 <= room < filled // 2


@gpu
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("runs", [1, 3])
def test_factor_gradients_of_overlapping_segments_stay_in_their_scratch(runs, dt):
    """The results mean nothing, but come from the scratch alone (what lies behind it is NaN) and are written to their place."""
    rows, segments, m, n, kmax = (OVERLAP[k] for k in ("rows", "segments", "m", "n", "kmax"))
    need = nmf.nmf_ragged_work_bytes(3, nmf.binding._TYPES[dt], rows, m, n, segments, runs, kmax, runs * kmax)
    mem = torch.full((64 * need // 4,), float("nan"), device="cuda")
    work = mem.view(torch.uint8)[:need]
    X, dY = torch.randn(rows, m, device="cuda").to(dt), torch.randn(rows, n, device="cuda").to(dt)
    U, V = torch.randn(rows, kmax, device="cuda"), torch.randn(rows, kmax, device="cuda")
    offsets = torch.tensor(overlapping(rows, segments), device="cuda")
    run = (torch.arange(segments, device="cuda") // 2 % runs).int()
    koff = (torch.arange(runs + 1, device="cuda") * kmax).int()
    outs = [torch.full((3 * runs * kmax, cols), 7.0, dtype=dt, device="cuda") for cols in (m, n)]
    dWt, dH = (o[runs * kmax:2 * runs * kmax] for o in outs)
    for scratch in (work, torch.empty(0, dtype=torch.uint8, device="cuda")):
        dWt.zero_(), dH.zero_()
        nmf.nmf_lowrank_gradient(X, dY, rows, m, n, offsets, run, segments, koff, runs, kmax, U, V, dWt, dH, work=scratch)
        torch.cuda.synchronize()
        assert bool(torch.isfinite(dWt.float()).all()) and bool(torch.isfinite(dH.float()).all())
        for o in outs:
            assert bool((o[:runs * kmax] == 7).all()) and bool((o[2 * runs * kmax:] == 7).all())
    assert bool(mem[need // 4:].isnan().all())


@pytest.mark.parametrize("rows,segments,kmax", [(512, 512, 64), (256, 256, 16), (4096, 40, 256)])
def test_scratch_of_factor_gradients_does_not_grow_with_idle_runs(rows, segments, kmax):
    """Only runs with several chunks have parts, and the rows bound their number."""
    need = [nmf.nmf_ragged_work_bytes(3, nmf.NMF_F32, rows, 8192, 8192, segments, runs, kmax, runs * kmax) for runs in (200, 2000, 8000)]
    assert need[0] == need[1] == need[2]
    assert nmf.nmf_ragged_work_bytes(3, nmf.NMF_F32, 60, 8192, 8192, 2, 2000, kmax, 2000 * kmax) == 0       # one chunk for each run


@gpu
@pytest.mark.parametrize("typ", ["f32", "bf16", "f16"])
def test_few_runs_with_many_rows_among_many_with_few(typ):
    """Three of 150 runs have several chunks, two of them behind the first 64; others one or none."""
    p = Problem(3000, 160, 150, 2, 40, 200, 136, False, typ)
    p.which[:50], p.which[60:75], p.which[100:140:2] = 70, 9, 149
    p.run = torch.tensor(p.which, dtype=torch.int32, device="cuda")
    Y, dX = torch.empty_like(p.dY), torch.empty_like(p.X)
    dWt, dH = torch.full_like(p.Wt, 5.0), torch.full_like(p.H, 5.0)
    p.forward(Y)
    p.backward(dX, dWt, dH)
    p.check_gradient(dWt, dH)


def parts(typ, rows, m, n, groups=1):
    """Parts that the contraction of a grouped product is cut into."""
    return max(1, nmf.nmf_ragged_work_bytes(0, typ, rows, m, n, groups) // (rows * n * 4))


def test_parts_of_products_go_by_what_they_cost_not_by_a_number_of_rows():
    """Long contractions of few tiles are split beyond 4096 rows as below; short ones of many rows are not, they would pay for the join."""
    for typ in (nmf.NMF_F32, nmf.NMF_BF16):
        assert parts(typ, 4096, 8192, 64) > 1 and parts(typ, 4097, 8192, 64) > 1 and parts(typ, 6000, 8192, 64) > 1
    assert parts(nmf.NMF_F32, 8192, 4096, 64, 64) > 1
    assert parts(nmf.NMF_BF16, 4096, 1024, 128) == 1 and parts(nmf.NMF_BF16, 4096, 512, 64) == 1
    assert parts(nmf.NMF_F32, 4096, 512, 256) == 1
    assert parts(nmf.NMF_BF16, 150, 4096, 1000) > 1 and parts(nmf.NMF_BF16, 24, 4096, 1000) > 1


@gpu
@pytest.mark.parametrize("typ", ["f32", "bf16", "f16"])
def test_products_of_many_rows_in_parts(typ):
    rows, m, n = 5003, 4096, 64
    dt = TYPES[typ]
    g = torch.Generator(device="cuda").manual_seed(3)
    X, B = torch.randn(rows, m, generator=g, device="cuda").to(dt), torch.randn(2, m, n, generator=g, device="cuda").to(dt)
    Y = torch.empty(rows, n, dtype=dt, device="cuda")
    cut = [0, 4100, rows]
    nmf.nmf_grouped_product(X, torch.tensor(cut, device="cuda"), 2, rows, B, False, m, n, Y)
    for i in range(2):
        x, b = X[cut[i]:cut[i + 1]].double(), B[i].double()
        within(Y[cut[i]:cut[i + 1]], x @ b, x.abs() @ b.abs(), m, typ)


@gpu
@pytest.mark.parametrize("typ", ["f32", "bf16", "f16"])
def test_gradients_of_more_groups_than_a_wave_has_lanes(typ):
    rows, groups, m, n = 900, 150, 136, 264
    dt = TYPES[typ]
    g = torch.Generator(device="cuda").manual_seed(4)
    X, dY = torch.randn(rows, m, generator=g, device="cuda").to(dt), torch.randn(rows, n, generator=g, device="cuda").to(dt)
    cut = lengths_of("ragged", rows, groups, 11)
    G = torch.full((groups, m, n), 5.0, dtype=dt, device="cuda")
    nmf.nmf_grouped_gradient(X, dY, torch.from_numpy(cut).cuda(), groups, rows, m, n, G)
    for i in range(groups):
        x, dy = X[cut[i]:cut[i + 1]].double(), dY[cut[i]:cut[i + 1]].double()
        within(G[i], x.t() @ dy, x.abs().t() @ dy.abs(), max(1, len(x)), typ)


def test_parts_of_lowrank_products_save_launches():
    """Few rows in long segments: the join of parts takes the adapters, which else are packed by a launch of their own."""
    def product_parts(typ, rows, m, n):
        room = nmf.nmf_ragged_work_bytes(2, typ, rows, m, n, 4, 2, 16, 32)
        return room // (rows * n * 4)                    # U packed is 128 bytes a row: less than one part of 128 columns

    assert product_parts(nmf.NMF_BF16, 300, 1024, 512) >= 4 and product_parts(nmf.NMF_BF16, 1000, 512, 128) >= 2
    assert product_parts(nmf.NMF_BF16, 4096, 512, 128) == 0 and product_parts(nmf.NMF_F32, 4096, 512, 128) == 0
    assert parts(nmf.NMF_BF16, 1000, 512, 128) == 1      # without adapters the join costs more than it saves

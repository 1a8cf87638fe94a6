"""Codes of 8 bits are the nearest ones to entry x 448 / largest (to entry x 2^126 in blocks whose scale is the smallest one).

Against that in 64 bits, without a tolerance: a quotient on the border between two codes has few bits, so 64 bits hold it, and
one of floats beside a border is 2^-48 of itself away from it at least, which 64 bits, off by 2^-53, tell apart.
"""
import pytest
import torch

import paper_2202_09518_amd as nmf

gpu = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
E8 = torch.float8_e4m3fn


def nearest(x, most):
    """Values of the codes of x (64 bits) in blocks whose largest magnitude is `most`."""
    q = torch.where(most > 448 * 2.0 ** -126, x * 448 / most, x * 2.0 ** 126)
    unit = torch.exp2((torch.frexp(q).exponent - 4).clamp_min(-9).double())
    return torch.round(q / unit) * unit


def on_borders(g, rows, low, high, dt):
    """Rows of 128 whose largest magnitude, the first entry, lies between 2^low and 2^high, and the others on borders of codes and beside."""
    most = torch.exp2(torch.randint(low, high, (rows, 1), generator=g, device="cuda").double()) * (1 + torch.rand(rows, 1, generator=g, device="cuda").double())
    most[::4] = 1.75 * torch.exp2(torch.randint(low, high, (rows // 4, 1), generator=g, device="cuda").double())      # quotients have few bits
    most = most.to(dt).double()
    fraction, exponent = torch.randint(8, 16, (rows, 128), generator=g, device="cuda"), torch.randint(-10, 6, (rows, 128), generator=g, device="cuda")
    border = (fraction + 0.5).double() * torch.exp2(exponent.double() - 1)
    x = (border * most.clamp_min(448 * 2.0 ** -126) / 448).to(dt)
    if dt is torch.float32:                                     # up to three last places beside
        x = (x.view(torch.int32) + torch.randint(-3, 4, (rows, 128), generator=g, device="cuda").int()).clamp_min(0).view(torch.float32)
    x = torch.minimum(x.double(), most) * (2 * torch.randint(0, 2, (rows, 128), generator=g, device="cuda") - 1)
    x[:, 0] = most[:, 0]
    assert bool((x.to(dt).double() == x).all())
    return x.to(dt)


@gpu
@pytest.mark.parametrize("typ", ["f32", "bf16"])
@pytest.mark.parametrize("low,high", [(-148, -120), (-124, -112), (-115, -90), (-70, -50), (100, 127)])
def test_codes_are_the_nearest_ones_at_the_ends_of_the_range(low, high, typ):
    g = torch.Generator(device="cuda").manual_seed(high)
    rows = 4096
    X = on_borders(g, rows, max(low, -132) if typ == "bf16" else low, high, TYPES[typ])
    for block in (1, 128):
        C, S = torch.empty(rows, 128, dtype=E8, device="cuda"), torch.empty(rows // block, 1, device="cuda")
        nmf.nmf_round_blocks(X, rows, 128, block, C, S)
        most = X.double().abs().view(rows // block, -1).amax(1, keepdim=True).repeat_interleave(block, 0)
        want = nearest(X.double(), most)
        bad = C.float().double() != want
        assert not bool(bad.any()), (block, int(bad.sum()), X[bad][:4], want[bad][:4], C.float()[bad][:4])


@gpu
@pytest.mark.parametrize("typ", ["f32", "bf16"])
@pytest.mark.parametrize("low,high", [(-124, -112), (-6, 7), (100, 126)])
@pytest.mark.parametrize("m", [128, 640, 4096, 9088, 32768])
def test_codes_of_the_norm_are_the_nearest_but_beside_borders(m, low, high, typ):
    """Rows of 1 and -1, whose norm is one: the weights come out as they are, on borders of codes and beside them.  Within 2^-22 of a border
    (scale, inverse and product are off by 2^-24 each) either neighbour will do."""
    g = torch.Generator(device="cuda").manual_seed(m)
    rows, dt = 5, TYPES[typ]
    w = on_borders(g, 256, low, high, dt).reshape(-1)[:m].contiguous()
    beside = torch.rand(m, generator=g, device="cuda") < 0.5               # some a little farther off
    beside[::128] = False
    w = torch.where(beside, w.double() * (1 - 2.0 ** -7), w.double()).to(dt)
    X = (2 * torch.randint(0, 2, (rows, m), generator=g, device="cuda") - 1).to(dt)
    Y, Y8, scale = torch.empty_like(X), torch.empty(rows, m, dtype=E8, device="cuda"), torch.empty(rows, m // 128, device="cuda")
    nmf.nmf_rms_norm(X, rows, m, 0.0, weight=w, Y=Y, Y8=Y8, scale=scale)
    assert torch.equal(Y, X * w)
    most = w.double().abs().view(-1, 128).amax(1)
    assert bool(((scale.double() - (most / 448).clamp_min(2.0 ** -126)).abs() <= scale.double() * 2.0 ** -24).all())
    y, most = Y.double(), most.repeat_interleave(128)[None]
    low, high = (nearest((y * (1 + s * 2.0 ** -22)).clamp(-most, most), most) for s in (-1, 1))
    got = Y8.float().double()
    assert bool(((got == low) | (got == high)).all())

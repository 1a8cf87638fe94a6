"""8-bit products of rows so long that distances inside a tile would pass 32 bits."""
import ctypes

import pytest
import torch

import paper_2202_09518_amd as nmf

gpu = pytest.mark.gpu
FAR = 2 ** 31 - 1                    # what one descriptor of a load straight to LDS reaches
AT = 4096                            # an address that is never touched
ROOM = 2 ** 40


def route(typ, rows, groups, m, n, transposed, one=False, ldx=None, ldb=None, first=0, work=ROOM):
    """Straight to LDS or not, bytes of copies, leading dimensions as the tiles read them, rows and columns of a tile, bytes of parts."""
    fn = nmf.lib().nmfmu_product8_route
    i32, i64, vp = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p
    fn.argtypes = [i32, vp, i64, i64, i32, i64, vp, i64, i64, i32, i64, i64, ctypes.c_size_t, ctypes.POINTER(i64)]
    out = (i64 * 7)()
    b_rows, b_cols = (n, m) if transposed else (m, n)
    ldx, ldb = ldx or m, ldb or b_cols
    assert fn(typ, AT + first, ldx, -(-m // 128), groups, rows, AT, ldb, 0 if one else b_rows * ldb, int(transposed), m, n, work, out) == nmf.NMF_OK
    return list(out)


SIZES = [16, 500, 4095, 4096, 2 ** 20 + 1, 2 ** 22 - 16, 2 ** 22 - 15, 2 ** 22 - 1, 2 ** 22, 2 ** 22 + 16, 2 ** 23 + 3, 2 ** 23 + 16, 17000001, 2 ** 25 + 1, 2 ** 31 - 1]


@pytest.mark.parametrize("typ", [nmf.NMF_F32, nmf.NMF_BF16])
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("odd", [0, 1])
def test_codes_that_go_straight_to_lds_stay_near(odd, transposed, typ):
    """The farthest byte of a tile from its first one, in the operands as they are read: copied or not."""
    some = [0, 0]
    for rows, groups in ((450, 8), (8192, 1), (20000, 3)):
        for m in SIZES:
            for n in SIZES:
                for pad in (0, 16, 2 ** 22):
                    b_cols = m if transposed else n
                    straight, copies, ldx, ldb, BM, BN, _ = route(typ, rows, groups, m, n, transposed, True, m + pad, b_cols + pad, odd)
                    some[straight] += 1
                    if straight:
                        assert (BM - 1) * ldx + 127 < FAR and ((BN if transposed else 128) - 1) * ldb + BN < FAR, (rows, m, n, pad)
                    else:
                        assert copies == 0
    assert some[0] and some[1]


@pytest.mark.parametrize("m,n,transposed", [(17000001, 450, True), (450, 17000001, False)])
def test_no_copies_are_asked_for_of_rows_that_far(m, n, transposed):
    layout = nmf.NMF_B_N_X_M if transposed else nmf.NMF_B_M_X_N
    for kind in (2 | layout, 2 | layout | nmf.NMF_ONE_B):
        assert nmf.nmf_routed_work_bytes(kind, 450, m, n, 8) == route(nmf.NMF_BF16, 450, 8, m, n, transposed, bool(kind & nmf.NMF_ONE_B))[6]


@gpu
def test_product8_of_rows_beyond_2_to_24():
    """450 rows of 17000001 codes, of which only the last 129 are not zero: the sums of those, in whole numbers that floats hold."""
    rows, groups, m, n = 450, 8, 17000001, 450
    g = torch.Generator(device="cuda").manual_seed(31)
    M, N, last = -(-m // 128), -(-n // 128), m - 129
    X, B = (torch.zeros(k, m, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for k in (rows, n))
    x, b = (torch.randint(-8, 9, (k, 129), generator=g, device="cuda").float() for k in (rows, n))
    X[:, last:], B[:, last:] = x.to(X.dtype), b.to(X.dtype)
    xs, bs = torch.ones(rows, M, device="cuda"), torch.ones(1, N, M, device="cuda")
    cut = torch.linspace(0, rows, groups + 1).long().cuda()
    Y = torch.empty(rows, n, device="cuda")
    nmf.nmf_grouped_product8(X, xs, cut, groups, rows, B[None].expand(groups, n, m), bs.expand(groups, N, M), True, m, n, Y)
    assert torch.equal(Y.double(), x.double() @ b.double().t().contiguous())

"""How far the 8-bit product reads where it loads chunks of 16 codes without a look at each: never behind its array's end.

(On the device this does not show: codes of columns that are not there are in no result, and the memory behind an array mostly
may be read.  So the kernel's own condition and addresses are followed on the host.)
"""
import ctypes

import pytest

import paper_2202_09518_amd as nmf


def reads(m, n, ld, c0, columns, k1):
    fn = nmf.lib().nmfmu_column_reads
    i64 = ctypes.c_int64
    fn.argtypes = [i64, i64, i64, i64, ctypes.c_int32, i64, ctypes.POINTER(i64)]
    out = (i64 * 2)()
    assert fn(m, n, ld, c0, columns, k1, out) == nmf.NMF_OK
    return out[0], out[1]


@pytest.mark.parametrize("columns", [64, 128])
def test_whole_stages_end_inside_the_array(columns):
    some = [0, 0]
    for m in (1, 127, 128, 129, 255, 256, 257, 300, 515):
        for n in [*range(1, 35), 63, 64, 65, 127, 128, 129, 130, 143, 200, 255, 257, 389]:
            for pad in (0, 1, 7, 15, 16, 40):
                ld = n + pad
                for c0 in range(0, n, columns):
                    for k1 in {m, min(m, 128), min(m, 384)}:                 # the whole contraction, or parts of it
                        stages, far = reads(m, n, ld, c0, columns, k1)
                        assert c0 + far <= (m - 1) * ld + n, (m, n, ld, c0, k1)
                        ends = [(k0 + 127) * ld + -(-min(n - c0, columns) // 16) * 16 for k0 in range(0, k1 - 127, 128)]
                        assert stages == sum(c0 + e <= (m - 1) * ld + n for e in ends)      # and none is left to the slower way for nothing
                        some[stages > 0] += 1
    assert some[0] and some[1]


def test_far_rows_are_looked_at_one_by_one():
    assert reads(300, 100, 2 ** 22 - 1, 0, 128, 300) == (2, 255 * (2 ** 22 - 1) + 112)
    assert reads(300, 100, 2 ** 22, 0, 128, 300) == (0, 0)

"""Block-scaled values and token scores without a GPU: the sizes of their arrays,
what the entry points refuse before they touch a device, and the reference that
the GPU tests compare with."""
import ctypes
import os

import numpy as np
import pytest

import paper_2608_11249_amd as dl
from mx_common import held, scale_exp

pytestmark = pytest.mark.skipif(not os.path.exists(dl.LIB_PATH), reason="libdlmc.so not built")


def sizes(fmt, rows, cols):
    a, b = ctypes.c_uint64(), ctypes.c_uint64()
    st = dl.lib().dlmc_mx_bytes(fmt, rows, cols, ctypes.byref(a), ctypes.byref(b))
    return st, a.value, b.value


@pytest.mark.parametrize("fmt,rows,cols,want", [
    (0, 1, 1, (128, 32 * 8)), (1, 1, 1, (256, 32 * 8)), (0, 33, 256, (33 * 128, 64 * 8)),
    (1, 32, 257, (32 * 512, 2 * 32 * 8)), (0, 126464, 4096, (126464 * 2048, 16 * 126464 * 8)),
    (1, 2 ** 31 - 1, 1 << 24, ((2 ** 31 - 1) << 24, 2 ** 31 * 8 << 16)), (0, 0, 100, (0, 0))])
def test_array_sizes(fmt, rows, cols, want):
    assert sizes(fmt, rows, cols) == (0,) + want


@pytest.mark.parametrize("fmt,rows,cols", [(2, 1, 1), (-1, 1, 1), (0, -1, 1), (0, 1, 0), (0, 1, (1 << 24) + 1)])
def test_array_sizes_refused(fmt, rows, cols):
    assert sizes(fmt, rows, cols)[0] == -1


def test_entry_points_refuse_a_null_model():
    L = dl.lib()
    calls = [
        (L.dlmc_mx_quantize, None, 0, 32, 1, 32, 0, None, None),
        (L.dlmc_mx_dequantize, None, None, 0, 1, 32, None, 0, 32),
        (L.dlmc_add_norm_mx, None, 0, 32, None, 0, 0, None, 0, None, 1, 1e-5, 1, 32, 1, None, None),
        (L.dlmc_mx_matmul, None, None, 1, None, None, 1, 1, 32, None, 0, 1),
        (L.dlmc_token_scores, None, 0, 8, 1, None, 0, None, None, None, None, None, 0),
    ]
    for fn, *args in calls:
        assert fn(None, *args) == -1
        assert b"NULL" in L.dlmc_last_error()
    n = ctypes.c_uint64()
    assert L.dlmc_token_scores_ws(None, 1, 0, ctypes.byref(n)) == -1


def test_reference_values():
    # every E2M1 value and every midpoint between two of them, ties to even, in a
    # block whose scale is 1 (its largest is 6)
    x = np.zeros((1, 32))
    x[0, :16] = [6, .25, .75, 1.25, 1.75, 2.5, 3.5, 5, -.25, -.75, 0.24, 0.26, 5.01, -4.99, .5, 3]
    want = [6, 0, 1, 1, 2, 2, 4, 4, 0, -1, 0, .5, 6, -4, .5, 3]
    assert np.array_equal(held(x, "fp4")[0, :16], want)
    assert scale_exp(x, "fp4")[0, 0] == 0
    x[0, 0] = np.nextafter(6, 7)
    assert scale_exp(x, "fp4")[0, 0] == 1
    y = np.full((1, 32), 448.0)
    assert scale_exp(y, "fp8")[0, 0] == 0 and np.array_equal(held(y, "fp8"), y)
    y[0, 1:4] = [2.0 ** -9, 2.0 ** -10, 17.0]
    assert np.array_equal(held(y, "fp8")[0, :4], [448, 2.0 ** -9, 0, 16])
    assert scale_exp(np.zeros((1, 32)), "fp8")[0, 0] == -127

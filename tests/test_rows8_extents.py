"""Matrices whose bytes would pass 64 bits are refused, so that the search for overlaps cannot be led astray.  Without a GPU: nothing is
launched."""
import ctypes

import pytest

from paper_2110_14871_b200 import build as gbuild
from paper_2110_14871_b200 import gdws

BASE, MOST = 1 << 30, (1 << 31) - 1024


@pytest.fixture(scope="module", autouse=True)
def built():
    gbuild.build_library()


def kernel_of(x, w, y):
    k = ctypes.c_int(-1)
    return gdws.lib().gdws_pointwise8_kernel(*(ctypes.addressof(a) for a in (x, w, y)), ctypes.byref(k))


def test_overlaps_of_matrices_that_pass_64_bits():
    """y lies in x in every call.  With 2^30 + 1 rows 2^34 bytes apart the distance of x's last row from its first is 2^64: zero, in 64 bits."""
    w = gdws.Rows8(BASE - (1 << 20), BASE - (1 << 22), 8, 64, 64)
    for rows, ld, message in (((1 << 30) + 1, 64, "overlap"), ((1 << 30) + 1, 1 << 34, "2^56"), (MOST, 1 << 38, "2^56")):
        y = gdws.Rows(BASE + (1 << 20), rows, 8, 8, gdws.BF16)
        assert kernel_of(gdws.Rows8(BASE, BASE * 64, rows, ld, 64), w, y) == gdws.ERR_INVALID_ARG and message in gdws.last_error(), gdws.last_error()


@pytest.mark.parametrize("rows,ld,fine", [(1 << 20, 1 << 36, True), ((1 << 20) + 1, 1 << 36, True), ((1 << 20) + 2, 1 << 36, False), (MOST, 1 << 25, True), (MOST, 1 << 26, False), (MOST, 1 << 38, False), (2, 1 << 38, True), (1, 1 << 62, True)])
def test_where_the_limit_lies(rows, ld, fine):
    x, w, y = gdws.Rows8(BASE, BASE << 33, rows, ld, 64), gdws.Rows8(BASE - (1 << 20), BASE - (1 << 22), 8, 64, 64), gdws.Rows(BASE << 30, rows, 8, 8, gdws.BF16)
    if fine:
        assert kernel_of(x, w, y) == gdws.OK, gdws.last_error()
    else:
        assert kernel_of(x, w, y) == gdws.ERR_INVALID_ARG and "2^56" in gdws.last_error()

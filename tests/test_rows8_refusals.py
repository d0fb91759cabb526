"""Arguments that the calls on rows refuse, and their message, without a GPU: nothing is launched for any of them."""
import ctypes

import pytest
import torch

from paper_2110_14871_b200 import build as gbuild
from paper_2110_14871_b200 import gdws

BASE = 1 << 30            # addresses that no refused call touches


@pytest.fixture(scope="module", autouse=True)
def built():
    gbuild.build_library()


def rows(ptr=BASE, n=4, ld=64, cols=64, dtype=gdws.BF16):
    return gdws.Rows(ptr, n, ld, cols, dtype)


def rows8(q=BASE * 2, scale=BASE * 3, n=4, ld=64, cols=64):
    return gdws.Rows8(q, scale, n, ld, cols)


def call(name, *args):
    refs = [ctypes.addressof(a) if isinstance(a, ctypes.Structure) else a for a in args]
    return getattr(gdws.lib(), name)(*refs)


BAD_ROWS = [dict(ptr=None), dict(ptr=BASE + 1), dict(n=-1), dict(n=1 << 31), dict(n=(1 << 31) - 1023), dict(cols=0), dict(cols=-3), dict(cols=(1 << 30) + 1, ld=1 << 31), dict(ld=63), dict(ld=-64), dict(dtype=2), dict(dtype=gdws.F32, ptr=BASE + 2)]
BAD_ROWS8 = [dict(q=None), dict(scale=None), dict(scale=BASE * 3 + 2), dict(n=-1), dict(n=(1 << 31) - 1023), dict(cols=0), dict(cols=(1 << 30) + 1, ld=1 << 31), dict(ld=63)]


@pytest.mark.parametrize("bad", BAD_ROWS)
def test_matrices(bad):
    w = rows8(BASE * 4, BASE * 5)
    assert call("gdws_quantize_rows", rows(**bad), rows8(), None) == gdws.ERR_INVALID_ARG and "gdws_quantize_rows: x" in gdws.last_error()
    assert call("gdws_dequantize_rows", rows8(), rows(**bad), None) == gdws.ERR_INVALID_ARG
    assert call("gdws_pointwise8", rows8(), w, None, 0, rows(**bad), None) == gdws.ERR_INVALID_ARG
    assert call("gdws_norm_quantize_rows", rows(**bad), None, None, None, 0, 1e-6, rows8(), None) == gdws.ERR_INVALID_ARG
    assert call("gdws_norm_quantize_rows", rows(), rows(**bad), None, None, 0, 1e-6, rows8(), None) == gdws.ERR_INVALID_ARG
    assert call("gdws_norm_quantize_rows", rows(), None, rows(**bad), None, 0, 1e-6, rows8(), None) == gdws.ERR_INVALID_ARG


@pytest.mark.parametrize("bad", BAD_ROWS8)
def test_matrices_in_8_bits(bad):
    w = rows8(BASE * 4, BASE * 5)
    assert call("gdws_quantize_rows", rows(), rows8(**bad), None) == gdws.ERR_INVALID_ARG
    assert call("gdws_norm_quantize_rows", rows(), None, None, None, 0, 1e-6, rows8(**bad), None) == gdws.ERR_INVALID_ARG
    assert call("gdws_dequantize_rows", rows8(**bad), rows(), None) == gdws.ERR_INVALID_ARG
    assert call("gdws_pointwise8", rows8(**bad), w, None, 0, rows(cols=4), None) == gdws.ERR_INVALID_ARG
    assert call("gdws_pointwise8", rows8(), rows8(**bad), None, 0, rows(cols=4), None) == gdws.ERR_INVALID_ARG and gdws.last_error()


def test_null_structures():
    w = rows8(BASE * 4, BASE * 5)
    for args in [("gdws_quantize_rows", None, rows8(), None), ("gdws_quantize_rows", rows(), None, None), ("gdws_dequantize_rows", None, rows(), None), ("gdws_dequantize_rows", rows8(), None, None),
                 ("gdws_norm_quantize_rows", None, None, None, None, 0, 1e-6, rows8(), None), ("gdws_norm_quantize_rows", rows(), None, None, None, 0, 1e-6, None, None),
                 ("gdws_pointwise8", None, w, None, 0, rows(cols=4), None), ("gdws_pointwise8", rows8(), None, None, 0, rows(cols=4), None), ("gdws_pointwise8", rows8(), w, None, 0, None, None)]:
        assert call(*args) == gdws.ERR_INVALID_ARG, args[0]


def test_shapes_that_do_not_fit():
    w = rows8(BASE * 4, BASE * 5, n=6)
    for args in [("gdws_quantize_rows", rows(n=5), rows8(), None), ("gdws_quantize_rows", rows(), rows8(cols=63), None), ("gdws_dequantize_rows", rows8(), rows(cols=32), None),
                 ("gdws_norm_quantize_rows", rows(), rows(BASE * 6, n=3), None, None, 0, 1e-6, rows8(), None), ("gdws_norm_quantize_rows", rows(), None, rows(BASE * 6, cols=32), None, 0, 1e-6, rows8(), None),
                 ("gdws_norm_quantize_rows", rows(), rows(BASE * 6, dtype=gdws.F32), None, None, 0, 1e-6, rows8(), None),
                 ("gdws_pointwise8", rows8(), rows8(BASE * 4, BASE * 5, cols=32), None, 0, rows(cols=4), None), ("gdws_pointwise8", rows8(), w, None, 0, rows(cols=5), None),
                 ("gdws_pointwise8", rows8(), w, None, 0, rows(n=3, cols=6), None), ("gdws_pointwise8", rows8(), rows8(BASE * 4, BASE * 5, n=0), None, 0, rows(cols=4), None),
                 ("gdws_pointwise8", rows8(), w, BASE * 7 + 2, 0, rows(cols=6), None)]:
        assert call(*args) == gdws.ERR_INVALID_ARG, args
    wide = dict(cols=131072, ld=131072)
    assert call("gdws_pointwise8", rows8(**wide), rows8(BASE * 4, BASE * 5, **wide), None, 0, rows(cols=4), None) == gdws.ERR_UNSUPPORTED


def test_norm_options():
    for eps in (0.0, -1.0, 1e-39, float("inf"), float("nan")):
        assert call("gdws_norm_quantize_rows", rows(), None, None, None, 0, eps, rows8(), None) == gdws.ERR_INVALID_ARG and "eps" in gdws.last_error()
    assert call("gdws_norm_quantize_rows", rows(), None, None, BASE * 7, 5, 1e-6, rows8(), None) == gdws.ERR_INVALID_ARG
    assert call("gdws_norm_quantize_rows", rows(), None, None, BASE * 7 + 2, gdws.F32, 1e-6, rows8(), None) == gdws.ERR_INVALID_ARG


def test_overlaps():
    x = rows()                                                             # 4 x 64 bf16: 512 bytes
    for q in (rows8(BASE + 500), rows8(BASE - 200), rows8(scale=BASE + 508), rows8(BASE * 2, BASE * 2 + 8)):
        assert call("gdws_quantize_rows", x, q, None) == gdws.ERR_INVALID_ARG and "overlap" in gdws.last_error()
        assert call("gdws_norm_quantize_rows", x, None, None, None, 0, 1e-6, q, None) == gdws.ERR_INVALID_ARG and "overlap" in gdws.last_error()
    assert call("gdws_norm_quantize_rows", x, None, None, BASE * 2 + 100, gdws.F32, 1e-6, rows8(), None) == gdws.ERR_INVALID_ARG
    # total: the same rows, or none of them
    for total in (rows(BASE + 2), rows(BASE, ld=65), rows(BASE * 2 - 64), rows(BASE * 3 - 2), rows(BASE * 7 - 128)):
        assert call("gdws_norm_quantize_rows", x, None, total, BASE * 7, gdws.F32, 1e-6, rows8(), None) == gdws.ERR_INVALID_ARG and "total" in gdws.last_error()
    for y in (rows(BASE * 2 + 200, ld=64), rows(BASE * 3 + 8)):
        assert call("gdws_dequantize_rows", rows8(), y, None) == gdws.ERR_INVALID_ARG and "overlap" in gdws.last_error()
    w = rows8(BASE * 4, BASE * 5, n=6)
    for ptr in (BASE * 2, BASE * 3 + 4, BASE * 4 + 100, BASE * 5 + 20, BASE * 7 + 8):
        assert call("gdws_pointwise8", rows8(), w, BASE * 7, 0, rows(ptr, cols=6), None) == gdws.ERR_INVALID_ARG and "overlap" in gdws.last_error()
    # columns of one buffer
    assert call("gdws_norm_quantize_rows", rows(ld=128), None, rows(BASE + 126, ld=128), None, 0, 1e-6, rows8(), None) == gdws.ERR_INVALID_ARG


@pytest.mark.parametrize("rows_,K,D,kernel", [
    (1, 4096, 4096, gdws.KERNEL8_FEW), (8, 512, 64, gdws.KERNEL8_FEW), (9, 512, 64, gdws.KERNEL8_SLICES), (16, 4096, 16384, gdws.KERNEL8_SLICES), (128, 1280, 256, gdws.KERNEL8_SLICES),
    (16384, 1280, 256, gdws.KERNEL8_PAIRS), (4096, 4096, 4096, gdws.KERNEL8_PAIRS), (0, 64, 64, gdws.KERNEL8_NONE)])
def test_kernel_of_a_call(rows_, K, D, kernel):
    """As a B200 chooses, by estimated time; rows that start anywhere do not go through TMA."""
    def choice(x, w, y):
        k = ctypes.c_int(-1)
        assert call("gdws_pointwise8_kernel", x, w, y, ctypes.byref(k)) == gdws.OK
        return k.value

    x, w, y = rows8(BASE, BASE * 3, rows_, K, K), rows8(BASE * 4, BASE * 5, D, K, K), rows(BASE * 6, rows_, D, D)
    assert choice(x, w, y) == kernel
    other = kernel if kernel in (gdws.KERNEL8_FEW, gdws.KERNEL8_NONE) else gdws.KERNEL8_ANY
    assert choice(rows8(BASE + 4, BASE * 3, rows_, K, K), w, y) == other
    assert choice(x, rows8(BASE * 4, BASE * 5, D, K + 1, K), y) == other
    assert call("gdws_pointwise8_kernel", x, w, y, None) == gdws.ERR_INVALID_ARG


def test_binding_refuses_what_is_not_on_the_current_device():
    x, q, s = torch.zeros((4, 8)), torch.zeros((4, 8), dtype=torch.int8), torch.zeros(4)
    for run in (lambda: gdws.quantize_rows(x, q, s), lambda: gdws.norm_quantize_rows(x, q, s), lambda: gdws.dequantize_rows(q, s, x), lambda: gdws.pointwise8(q, s, q, s, torch.zeros((4, 4)))):
        with pytest.raises(ValueError):
            run()

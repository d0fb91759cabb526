"""gdws_pointwise8 uses nothing but its operands' elements: rows, weights, scales and bias among NaN, infinities and the largest steps."""
import pytest
import torch

from paper_2110_14871_b200 import build as gbuild
from paper_2110_14871_b200 import gdws

from rows8_util import HALF, product_of
from test_gpu_pointwise8 import TYPES, ceil16
from test_gpu_rows8_neighbours import Among, among

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    gbuild.build_library()


def operand(rows, cols, seed, around, ld, shift, vshift):
    """8-bit rows and their scales, each among values that spoil a sum."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    q = Among(torch.randint(-128, 128, (rows, cols), generator=gen, device="cuda").to(torch.int8), around, ld, shift)
    return q, Among(torch.rand((1, rows), generator=gen, device="cuda") * 0.02 + 1e-4, around, None, vshift)


@pytest.mark.parametrize("around", ["nan", "inf"])
@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("rows,K,D,aligned,kernel", [
    (1, 37, 5, True, gdws.KERNEL8_FEW), (1, 1203, 301, False, gdws.KERNEL8_FEW), (2, 513, 66, True, gdws.KERNEL8_FEW), (3, 100, 129, False, gdws.KERNEL8_FEW), (7, 2049, 131, True, gdws.KERNEL8_FEW),
    (40, 3001, 300, True, gdws.KERNEL8_SLICES), (130, 100, 127, True, gdws.KERNEL8_SLICES), (17, 33, 1001, True, gdws.KERNEL8_SLICES), (2561, 1001, 2601, True, gdws.KERNEL8_PAIRS),
    (9, 37, 65, False, gdws.KERNEL8_ANY), (70, 1203, 130, False, gdws.KERNEL8_ANY)])
def test_every_kernel(rows, K, D, aligned, kernel, out, around):
    for shift, vshift in ((0, 0), (0, 3), (1, 1)) if not aligned else ((0, 0), (0, 1), (16, 2)):
        ld = ceil16(K) + 16 if aligned else K
        x, xs = operand(rows, K, 1, around, ld, shift, vshift)
        w, ws = operand(D, K, 2, around, ld, shift, vshift)
        bias = Among(torch.randn((1, D), device="cuda", generator=torch.Generator(device="cuda").manual_seed(3)), around, None, vshift)
        y = among((rows, D), TYPES[out], around, D + vshift, vshift)
        assert gdws.pointwise8_kernel(x.t, xs.t[0], w.t, ws.t[0], y.t) == kernel
        gdws.pointwise8(x.t, xs.t[0], w.t, ws.t[0], y.t, bias=bias.t[0])
        gdws.rows_status()
        want, bound = product_of(x.t, xs.t[0], w.t, ws.t[0], bias.t[0], False)
        if out == "bf16":
            bound = bound + HALF[torch.bfloat16] * (want.abs() + bound)
        assert ((y.t.double() - want).abs() <= bound).all(), (shift, vshift)
        for f, name in ((x, "x"), (xs, "x's scales"), (w, "w"), (ws, "w's scales"), (bias, "the bias"), (y, "y")):
            f.check(name)

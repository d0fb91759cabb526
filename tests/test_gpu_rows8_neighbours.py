"""The calls on rows use nothing but their operands' elements: every operand lies in memory that holds NaN or infinity (8-bit ones:
-1 or -128) wherever it holds no element, on a boundary of 16 bytes and off it."""
import pytest
import torch

from paper_2110_14871_b200 import build as gbuild
from paper_2110_14871_b200 import gdws

from rows8_util import Field, steps_of
from test_gpu_rows8 import TYPES, norm_bound, values

pytestmark = pytest.mark.gpu

AROUND = {"nan": float("nan"), "inf": float("inf")}


@pytest.fixture(scope="module", autouse=True)
def built():
    gbuild.build_library()


class Among(Field):
    """A matrix among values that spoil every sum and maximum they get into."""

    def __init__(self, x, around, ld=None, shift=0):
        super().__init__(x.shape[0], x.shape[1], x.dtype, ld, shift)
        self.flat.fill_(AROUND[around] if x.dtype.is_floating_point else {"nan": -1, "inf": -128}[around])
        self.t.copy_(x)
        self.before = self.raw.clone()

    def check(self, what):
        assert torch.equal(self.raw[self.outside], self.before[self.outside]), f"bytes around {what} were overwritten"


def among(shape, dtype, around, ld=None, shift=0):
    return Among(torch.zeros(shape, dtype=dtype, device="cuda"), around, ld, shift)


# 65 to 20003: the kernels of rows that start anywhere, from two threads a row on, each with 1, 2 and 3 columns beyond a multiple of four
@pytest.mark.parametrize("around", ["nan", "inf"])
@pytest.mark.parametrize("wtype", ["f32", "bf16"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cols", [33, 65, 66, 67, 101, 250, 511, 763, 1001, 1531, 2047, 4091, 8190, 16381, 20003, 33001])
def test_norm(cols, dtype, wtype, around):
    rows, eps = 5, 1e-5
    x, r = values(rows, cols, dtype, cols), values(rows, cols, dtype, cols + 1)
    w = (1 + 0.3 * values(1, cols, "f32", 5)).to(TYPES[wtype])
    h = x.float() + r.float()
    u = h * w.float()
    want = steps_of(u)[0]
    want_scale = u.double().abs().amax(1) / 127 / torch.sqrt(h.double().square().mean(1) + eps)
    for gap, shift, wshift in ((0, 0, 0), (0, 1, 0), (0, 0, 1), (3, 2, 0), (8 - cols % 8, 0, 0), (8 - cols % 8, 3, 2)):
        fx, fr, fw = (Among(v, around, v.shape[1] + g, s) for v, g, s in ((x, gap, shift), (r, gap, shift), (w, 0, wshift)))
        total, q, scale = among((rows, cols), TYPES[dtype], around, cols + gap, shift), among((rows, cols), torch.int8, around, cols + gap, shift), among((1, rows), torch.float32, around)
        gdws.norm_quantize_rows(fx.t, q.t, scale.t[0], weight=fw.t[0], eps=eps, residual=fr.t, total=total.t)
        assert torch.equal(q.t, want) and torch.equal(total.t, h.to(TYPES[dtype])), (gap, shift, wshift)
        assert ((scale.t[0].double() - want_scale).abs() <= norm_bound(cols) * want_scale).all(), (gap, shift, wshift)
        for f, name in ((fx, "x"), (fr, "the residual"), (fw, "the weight"), (total, "total"), (q, "q"), (scale, "the scales")):
            f.check(name)


@pytest.mark.parametrize("around", ["nan", "inf"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cols", [1, 7, 30, 66, 250, 511, 763, 1001, 1531, 4091, 16381, 33001])
def test_quantize_and_back(cols, dtype, around):
    rows = 5
    x = values(rows, cols, dtype, cols)
    want, want_scale = steps_of(x.float())
    for gap, shift in ((0, 0), (0, 1), (3, 2), (8 - cols % 8, 0)):
        fx = Among(x, around, cols + gap, shift)
        q, scale, y = among((rows, cols), torch.int8, around, cols + gap, shift), among((1, rows), torch.float32, around), among((rows, cols), TYPES[dtype], around, cols + gap, shift)
        gdws.quantize_rows(fx.t, q.t, scale.t[0])
        assert torch.equal(q.t, want) and torch.equal(scale.t[0], want_scale), (gap, shift)
        gdws.dequantize_rows(q.t, scale.t[0], y.t)
        assert torch.equal(y.t, (want.float() * want_scale[:, None]).to(TYPES[dtype])), (gap, shift)
        for f, name in ((fx, "x"), (q, "q"), (scale, "the scales"), (y, "y")):
            f.check(name)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_weight_that_is_not_finite_still_counts(dtype):
    """Zeroing what lies behind the weight spares the weight's own infinities and NaN."""
    for cols in (101, 1531):
        x = values(4, cols, dtype, 3)
        for bad in (float("inf"), float("nan")):
            for at in (0, cols // 2, cols - 1):
                w = torch.ones((1, cols), device="cuda")
                w[0, at] = bad
                q, scale = gdws.empty_rows8(4, cols)
                gdws.norm_quantize_rows(x, q, scale, weight=Among(w, "nan").t[0])
                assert torch.isnan(scale).all() and not q.any()

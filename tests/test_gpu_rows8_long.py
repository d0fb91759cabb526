"""Long rows: the sum of squares keeps its bits however many there are."""
import pytest
import torch

from paper_2110_14871_b200 import build as gbuild
from paper_2110_14871_b200 import gdws

from rows8_util import Field, steps_of
from test_gpu_rows8 import TYPES, values

pytestmark = pytest.mark.gpu

# A square and its sum over a thread (64 bits) are rounded to fp32, ten additions join the threads' sums; the square root halves these
# twelve, the division by the columns, the columns themselves and eps.  Root, m / 127 and the quotient: one each.  10.5 steps.
BOUND = 11 * 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def built():
    gbuild.build_library()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("value", [1.1015625, 0.30078125, 5e-3])
@pytest.mark.parametrize("rows,cols", [(2, 40000), (1, 1000001), (1, 1 << 24)])
def test_equal_values(rows, cols, value, dtype):
    """The worst for a running sum: every addition is rounded the same way."""
    x = torch.full((rows, cols), value, device="cuda", dtype=TYPES[dtype])
    q, scale = gdws.empty_rows8(rows, cols)
    gdws.norm_quantize_rows(x, q, scale, eps=1e-6)
    h = x.double()
    want = h.amax(1) / 127 / torch.sqrt(h.square().mean(1) + 1e-6)
    assert ((scale.double() - want).abs() <= BOUND * want).all() and (q == 127).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cols", [33001, 131071, 500000])
def test_values_residual_and_weight(cols, dtype):
    rows = 3
    x, r = values(rows, cols, dtype, cols), values(rows, cols, dtype, cols + 1)
    x[1] *= 100
    w = 1 + 0.3 * values(1, cols, "f32", 5)[0]
    h = x.float() + r.float()
    q, scale, total = Field(rows, cols, torch.int8), Field(1, rows, torch.float32), Field(rows, cols, TYPES[dtype])
    gdws.norm_quantize_rows(x, q.t, scale.t[0], weight=w, eps=1e-5, residual=r, total=total.t)
    assert torch.equal(q.t, steps_of(h * w)[0]) and torch.equal(total.t, h.to(TYPES[dtype]))
    want = (h * w).double().abs().amax(1) / 127 / torch.sqrt(h.double().square().mean(1) + 1e-5)
    assert ((scale.t[0].double() - want).abs() <= BOUND * want).all()
    for f in (q, scale, total):
        f.check("a matrix")


def test_squares_that_pass_fp32_only_together():
    """Each square fits fp32 (3.4028e38); their sums are 4e40 and 4e38, which do not: NaN, as in shorter rows; and 3.24e38, which does."""
    cols = 40000
    x = torch.full((3, cols), 1e18, device="cuda")
    x[1], x[2] = 1e17, 9e16
    q, scale = gdws.empty_rows8(3, cols)
    gdws.norm_quantize_rows(x, q, scale)
    assert torch.isnan(scale[:2]).all() and not q[:2].any() and torch.isfinite(scale[2]) and (q[2] == 127).all()

"""What the calls on rows report when a wait inside a kernel runs out."""
import pytest
import torch

from paper_2110_14871_b200 import build as gbuild
from paper_2110_14871_b200 import gdws

from rows8_util import product_of
from test_gpu_rows8 import values

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    gbuild.build_library()


def test_a_wait_that_runs_out_is_reported_once():
    """The kernel returns by itself; the status is reported, cleared, and the calls go on."""
    gdws.rows_status()
    gdws.rows_selftest_wait(polls=32)
    with pytest.raises(gdws.GdwsError) as e:
        gdws.rows_status()
    assert e.value.status == gdws.ERR_DEVICE_TIMEOUT
    gdws.rows_status()
    with pytest.raises(gdws.GdwsError) as e:
        gdws.rows_selftest_wait(polls=65537)
    assert e.value.status == gdws.ERR_INVALID_ARG
    for rows, k, d in ((3, 256, 64), (40, 512, 200), (600, 512, 600)):
        q, scale = gdws.empty_rows8(rows, k)
        w, w_scale = gdws.empty_rows8(d, k)
        gdws.quantize_rows(values(rows, k, "f32", 1), q, scale)
        gdws.quantize_rows(values(d, k, "f32", 2), w, w_scale)
        y = torch.empty((rows, d), device="cuda")
        gdws.pointwise8(q, scale, w, w_scale, y)
        want, bound = product_of(q, scale, w, w_scale, None, False)
        assert ((y.double() - want).abs() <= bound).all()
    gdws.rows_status()

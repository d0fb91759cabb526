"""Calls on rows left to another stream; norms of the widest rows that one block keeps in registers."""
import pytest
import torch

from paper_2110_14871_b200 import build as gbuild
from paper_2110_14871_b200 import gdws

from rows8_util import Field, product_of, steps_of
from test_gpu_rows8 import TYPES, norm_bound, values

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    gbuild.build_library()


def test_the_order_on_another_stream():
    """Every output is spoiled on the side stream before the calls there, so that nothing of the first pass is left."""
    x, r = values(50, 1000, "bf16", 21), values(50, 1000, "bf16", 22)
    q, scale = gdws.empty_rows8(50, 1000)
    w, w_scale = gdws.empty_rows8(72, 1000)
    gdws.quantize_rows(values(72, 1000, "f32", 3), w, w_scale)
    total, y, z = torch.empty_like(x), torch.empty_like(x), torch.empty((50, 72), device="cuda")

    def step():
        gdws.norm_quantize_rows(x, q, scale, residual=r, total=total)
        gdws.dequantize_rows(q, scale, y)
        gdws.pointwise8(q, scale, w, w_scale, z)

    step()
    want = [t.clone() for t in (q, scale, total, y, z)]
    assert torch.equal(want[0], steps_of(x.float() + r.float())[0])
    for stream in (torch.cuda.Stream(), torch.cuda.Stream(priority=-1)):
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            for t in (scale, total, y, z):
                t.fill_(float("nan"))
            q.fill_(99)
            step()
        torch.cuda.current_stream().wait_stream(stream)
        assert all(torch.equal(a, b) for a, b in zip((q, scale, total, y, z), want))


@pytest.mark.parametrize("operands", ["all", "x"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols,gap,shift", [(3, 16392, 0, 0), (2, 20000, 8, 0), (300, 24576, 0, 0), (2, 32760, 0, 0), (3, 32768, 0, 0), (150, 32761, 7, 0), (3, 16386, 0, 0), (2, 32761, 0, 1), (3, 24999, 0, 0), (2, 32768, 1, 1)])
def test_norms_of_wide_rows(rows, cols, gap, shift, dtype, operands):
    """Rows that start on 16 bytes and elsewhere, their registers full: 32 values a thread, and what is added to them."""
    x = Field(rows, cols, TYPES[dtype], cols + gap, shift)
    x.t.copy_(values(rows, cols, dtype, cols))
    r = w = total = None
    if operands == "all":
        r, total = Field(rows, cols, TYPES[dtype], cols + gap, shift), Field(rows, cols, TYPES[dtype], cols + gap, shift)
        r.t.copy_(3 * values(rows, cols, dtype, cols + 1))
        w = 1 + 0.3 * values(1, cols, "f32", 5)[0]
    h = x.t.float() + r.t.float() if r else x.t.float()
    u = h * w if r else h
    q, scale = Field(rows, cols, torch.int8, cols + gap, shift), Field(1, rows, torch.float32)
    gdws.norm_quantize_rows(x.t, q.t, scale.t[0], weight=w, eps=1e-5, residual=r.t if r else None, total=total.t if r else None)
    assert torch.equal(q.t, steps_of(u)[0])
    want = u.double().abs().amax(1) / 127 / torch.sqrt(h.double().square().mean(1) + 1e-5)
    assert ((scale.t[0].double() - want).abs() <= norm_bound(cols) * want).all()
    if r:
        assert torch.equal(total.t, h.to(TYPES[dtype]))
    for f in (x, r, total, q, scale):
        if f:
            f.check("a matrix")


def test_streams_given_to_the_calls():
    """stream=: an object or a handle; the work is ordered there, behind what fills its inputs late."""
    w, w_scale = gdws.empty_rows8(72, 1000)
    gdws.quantize_rows(values(72, 1000, "f32", 3), w, w_scale)
    late, gain = values(400, 1000, "bf16", 4), torch.nn.Parameter(torch.ones(1000, device="cuda"))
    for given in (lambda s: s, lambda s: s.cuda_stream):
        s = torch.cuda.Stream()
        x, r = torch.zeros((400, 1000), dtype=torch.bfloat16, device="cuda"), values(400, 1000, "bf16", 5)
        q, scale = gdws.empty_rows8(400, 1000)
        total, y, z = torch.empty_like(x), torch.empty_like(x), torch.empty((400, 72), device="cuda")
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            torch.cuda._sleep(2_000_000)                # about a millisecond
            x.copy_(late)
        gdws.norm_quantize_rows(x, q, scale, weight=gain, residual=r, total=total, stream=given(s))
        gdws.dequantize_rows(q, scale, y, stream=given(s))
        gdws.pointwise8(q, scale, w, w_scale, z, stream=given(s))
        torch.cuda.current_stream().wait_stream(s)
        h = late.float() + r.float()
        assert torch.equal(q, steps_of(h)[0]) and torch.equal(total, h.bfloat16()) and torch.equal(y, (q.float() * scale[:, None]).bfloat16())
        want, bound = product_of(q, scale, w, w_scale, None, False)
        assert ((z.double() - want).abs() <= bound).all()

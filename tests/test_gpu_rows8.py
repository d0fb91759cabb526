"""gdws_quantize_rows, gdws_norm_quantize_rows and gdws_dequantize_rows against their definitions in 64 bits: every q equal, sums
of squares within the rounding of their fp32 additions, nothing written beside the rows."""
import os
import subprocess
import sys

import pytest
import torch

from paper_2110_14871_b200 import build as gbuild
from paper_2110_14871_b200 import gdws

from rows8_util import HALF, Field, steps_of

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module", autouse=True)
def built():
    gbuild.build_library()


def values(rows, cols, dtype, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((rows, cols), generator=gen, device="cuda")
    x *= torch.where(torch.rand(cols, generator=gen, device="cuda") < 0.02, 15.0, 1.0)
    return x.to(TYPES[dtype])


def field_of(x, ld=None, shift=0):
    f = Field(x.shape[0], x.shape[1], x.dtype, ld, shift)
    f.t.copy_(x)
    return f


# rows, cols; (extra elements between rows, first element's shift) of x and of q
SHAPES = [(1, 1), (3, 7), (9, 64), (5, 256), (33, 257), (2, 512), (7, 513), (4, 1337), (3, 2048), (2, 2049), (1, 4096), (3, 4097), (2, 8192),
          (2, 8193), (1, 16384), (2, 16391), (1, 32768), (2, 32769), (1, 70001)]
GAPS = [((0, 0), (0, 0)), ((8, 0), (16, 0)), ((1, 0), (3, 1)), ((0, 1), (0, 0))]


@pytest.mark.parametrize("gaps", range(len(GAPS)))
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_quantize(rows, cols, dtype, gaps):
    (gx, sx), (gq, sq) = GAPS[gaps]
    x = field_of(values(rows, cols, dtype, 7 * rows + cols), cols + gx, sx)
    q, scale, y = Field(rows, cols, torch.int8, cols + gq, sq), Field(1, rows, torch.float32), Field(rows, cols, TYPES[dtype], cols + gx, sx)
    gdws.quantize_rows(x.t, q.t, scale.t[0])
    gdws.dequantize_rows(q.t, scale.t[0], y.t)
    torch.cuda.synchronize()
    want, want_scale = steps_of(x.t.float())
    assert torch.equal(q.t, want) and torch.equal(scale.t[0], want_scale)
    assert torch.equal(y.t, (want.float() * want_scale[:, None]).to(TYPES[dtype]))
    for f, name in ((x, "x"), (q, "q"), (scale, "the scales"), (y, "y")):
        f.check(name)


def norm_bound(cols):
    """Relative: a thread adds up at most max(32, cols / 1024 + 1) squares, ten additions join the threads' sums; the square root
    halves what that amounts to.  Division by cols, eps, root, m / 127 and the quotient: five roundings."""
    return ((max(32, cols // 1024 + 1) + 10) / 2 + 5.5) * 2.0 ** -24


@pytest.mark.parametrize("residual,total,weight", [(True, "own", "f32"), (True, "residual", "bf16"), (False, None, "f32"), (True, "x", None), (False, "own", "bf16"), (True, None, "f32")])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols,gap,shift", [(1, 1, 0, 0), (5, 96, 0, 0), (9, 333, 0, 0), (300, 512, 8, 0), (3, 1536, 0, 0), (2, 2049, 7, 1), (2, 4096, 0, 0), (2, 8191, 0, 0), (1, 16384, 0, 0), (2, 33000, 0, 0),
                                                 (1, 40001, 0, 1)])
def test_norm_quantize(rows, cols, gap, shift, dtype, residual, total, weight):
    eps = 1e-5
    x = field_of(values(rows, cols, dtype, rows + cols), cols + gap, shift)
    r = field_of(3 * values(rows, cols, dtype, rows + cols + 1), cols + gap, shift) if residual else None
    w = (1 + 0.3 * values(1, cols, "f32", 5)[0]).to(TYPES[weight]) if weight else None
    h = x.t.float() + r.t.float() if residual else x.t.float()
    u = h * w.float() if weight else h
    t = {None: None, "own": Field(rows, cols, TYPES[dtype], cols + gap, shift), "residual": r, "x": x}[total]
    q, scale = Field(rows, cols, torch.int8, cols + gap, shift), Field(1, rows, torch.float32)
    gdws.norm_quantize_rows(x.t, q.t, scale.t[0], weight=w, eps=eps, residual=r.t if residual else None, total=t.t if t else None)
    torch.cuda.synchronize()
    want, _ = steps_of(u)
    assert torch.equal(q.t, want)
    want_scale = u.double().abs().amax(1) / 127 / torch.sqrt(h.double().square().mean(1) + eps)
    assert ((scale.t[0].double() - want_scale).abs() <= norm_bound(cols) * want_scale).all()
    if t:
        assert torch.equal(t.t, h.to(TYPES[dtype]))
    for f in (x, r, t, q, scale):
        if f:
            f.check("a matrix")


@pytest.mark.parametrize("odd", [0, 1])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cols", [16, 32, 56, 120, 240, 440, 700, 960, 1240, 1496, 1960, 2960, 4064, 6000, 8000, 12000, 16000])
def test_more_rows_than_fill_the_chip(cols, dtype, odd):
    """As many rows as take the threads per row that large calls do; the last block has a row too few."""
    cols += odd
    rows = 2_600_000 // cols + 3
    x, r = values(rows, cols, dtype, cols), values(rows, cols, dtype, cols + 1)
    w = 1 + 0.2 * values(1, cols, "f32", 3)[0]
    q, scale = Field(rows, cols, torch.int8, (cols + 15) // 16 * 16), Field(1, rows, torch.float32)
    total, y = Field(rows, cols, TYPES[dtype]), Field(rows, cols, TYPES[dtype])
    gdws.quantize_rows(x, q.t, scale.t[0])
    want, want_scale = steps_of(x.float())
    assert torch.equal(q.t, want) and torch.equal(scale.t[0], want_scale)
    gdws.norm_quantize_rows(x, q.t, scale.t[0], weight=w, residual=r, total=total.t)
    h = x.float() + r.float()
    assert torch.equal(q.t, steps_of(h * w)[0]) and torch.equal(total.t, h.to(TYPES[dtype]))
    want_scale = (h * w).double().abs().amax(1) / 127 / torch.sqrt(h.double().square().mean(1) + 1e-6)
    assert ((scale.t[0].double() - want_scale).abs() <= norm_bound(cols) * want_scale).all()
    gdws.dequantize_rows(q.t, scale.t[0], y.t)
    assert torch.equal(y.t, (q.t.float() * scale.t[0][:, None]).to(TYPES[dtype]))
    for f in (q, scale, total, y):
        f.check("a matrix")


@pytest.mark.parametrize("cols", [5, 61, 130, 1000, 1333, 5003, 20001])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_matrices_that_lie_differently(dtype, cols):
    """x, residual and total each at another place within 16 bytes, the weight off its boundary, q at every place."""
    x, r = values(5, cols, dtype, cols), values(5, cols, dtype, cols + 1)
    w = Field(1, cols, torch.float32, None, 1)
    w.t.copy_(1 + 0.2 * values(1, cols, "f32", 3))
    for sx, sr, st in ((0, 1, 2), (3, 3, 3), (1, 1, 1)):
        fx, fr, ft, scale = field_of(x, cols + 1, sx), field_of(r, cols + (1 if sx == sr else 2), sr), Field(5, cols, TYPES[dtype], cols + 1, st), Field(1, 5, torch.float32)
        for sq in range(8):
            q = Field(5, cols, torch.int8, cols + sq, sq)
            gdws.norm_quantize_rows(fx.t, q.t, scale.t[0], weight=w.t[0], residual=fr.t, total=ft.t)
            h = x.float() + r.float()
            assert torch.equal(q.t, steps_of(h * w.t)[0]) and torch.equal(ft.t, h.to(TYPES[dtype]))
            y = Field(5, cols, TYPES[dtype], cols + 3, sq)
            gdws.dequantize_rows(q.t, scale.t[0], y.t)
            assert torch.equal(y.t, (q.t.float() * scale.t[0][:, None]).to(TYPES[dtype]))
            for f in (fx, fr, ft, q, y, scale, w):
                f.check("a matrix")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_halfway_cases(dtype):
    """Quotients that lie exactly between two integers, and next to it."""
    u = torch.arange(-254, 255, device="cuda").float() / 2          # with 127 in the row: every second one is a tie
    u = torch.stack([torch.cat([u, torch.tensor([127.0], device="cuda")]), torch.cat([u * 2 ** -9, torch.tensor([127.0 * 2 ** -9], device="cuda")])])
    x = u.to(TYPES[dtype])
    assert torch.equal(x.float(), u)
    if dtype == "f32":      # one step of the type beside the ties
        x = torch.cat([x, torch.nextafter(x, torch.full_like(x, 1e9)).clamp(-127, 127), torch.nextafter(x, torch.full_like(x, -1e9)).clamp(-127, 127)])
    q, scale = gdws.empty_rows8(*x.shape)
    gdws.quantize_rows(x, q, scale)
    assert torch.equal(q, steps_of(x.float())[0])
    x = values(64, 4096, dtype, 3)
    x[:, ::5] = x.abs().amax(1, keepdim=True) / 2                     # 63.5 steps
    q, scale = gdws.empty_rows8(*x.shape)
    gdws.quantize_rows(x, q, scale)
    assert torch.equal(q, steps_of(x.float())[0])


def test_every_pair_of_bf16_significands():
    """127 u / m for all 8-bit significands of u and m and nine binades of u: ties and what lies nearest to them."""
    u = torch.cat([torch.arange(128, 256, device="cuda").float() * 2.0 ** -k for k in range(9)])
    for m in range(128, 256):
        row = torch.cat([u[u <= m], torch.tensor([float(m)], device="cuda")])
        x = torch.stack([row, -row, row * 2.0 ** 100, row * 2.0 ** -100, row * 2.0 ** -130]).bfloat16()
        q, scale = gdws.empty_rows8(*x.shape)
        for run in (gdws.quantize_rows, gdws.norm_quantize_rows):
            if run is gdws.norm_quantize_rows:
                x = x[[0, 1, 3, 4]].contiguous()                 # 2^100 squared passes fp32
                q, scale = gdws.empty_rows8(*x.shape)
            run(x, q, scale)
            assert torch.equal(q, steps_of(x.float())[0]), m


def test_neighbours_of_ties_in_fp32():
    gen = torch.Generator(device="cuda").manual_seed(9)
    for ulps in range(-3, 4):
        m = torch.rand((64, 1), generator=gen, device="cuda") * 2.0 ** torch.randint(-20, 20, (64, 1), generator=gen, device="cuda").float() + 1e-6
        u = (torch.randint(0, 127, (64, 500), generator=gen, device="cuda").float() + 0.5) * m / 127
        for _ in range(abs(ulps)):
            u = torch.nextafter(u, torch.full_like(u, float("inf") if ulps > 0 else -float("inf")))
        x = torch.cat([torch.minimum(u, m), -torch.minimum(u, m), m], 1)
        q, scale = gdws.empty_rows8(*x.shape)
        for run in (gdws.quantize_rows, gdws.norm_quantize_rows):
            run(x, q, scale)
            assert torch.equal(q, steps_of(x)[0])


@pytest.mark.parametrize("cols", [5, 256, 1000, 4096, 40000])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_zero_tiny_huge_and_not_finite(dtype, cols):
    x = values(9, cols, dtype, 11)
    x[0] = 0
    x[1] *= 2.0 ** -120
    x[2] = x[2].float().mul(2.0 ** -100).mul(2.0 ** -40).to(x.dtype)      # subnormal in either type
    x[3] = (x[3].float() / x[3].float().abs().max()).to(x.dtype) * 2.0 ** 127
    x[4, cols // 2] = float("inf")
    x[5, cols - 1] = float("-inf")
    x[6, 0] = float("nan")
    x[7] = -0.0
    w = torch.ones(cols, device="cuda")
    for norm in (False, True):
        q, scale = gdws.empty_rows8(9, cols)
        if norm:
            gdws.norm_quantize_rows(x, q, scale, weight=w)
        else:
            gdws.quantize_rows(x, q, scale)
        want, want_scale = steps_of(x.float())
        if norm:
            want[3], want_scale[3] = 0, float("nan")                      # its squares pass fp32
        assert torch.equal(q, want)
        assert torch.equal(torch.isnan(scale), torch.isnan(want_scale)) and scale[0] == 0 and scale[7] == 0
        if not norm:
            assert torch.equal(scale.nan_to_num(-1), want_scale.nan_to_num(-1))
        y = torch.empty((9, cols), device="cuda")
        gdws.dequantize_rows(q, scale, y)
        assert torch.isnan(y[4:7]).all() and not torch.isnan(y[:3]).any() and (y[0] == 0).all()


def test_no_rows_and_views():
    q, scale = gdws.empty_rows8(0, 40)
    gdws.quantize_rows(torch.empty((0, 40), device="cuda"), q, scale)
    gdws.norm_quantize_rows(torch.empty((0, 40), device="cuda"), q, scale)
    gdws.dequantize_rows(q, scale, torch.empty((0, 40), device="cuda"))
    # an NHWC map is rows of channels; x and total as columns of one buffer
    x = values(2 * 5 * 3, 24, "bf16", 2)
    qa, sa = torch.empty((2, 5, 3, 24), dtype=torch.int8, device="cuda"), torch.empty(30, device="cuda")
    gdws.quantize_rows(x.view(2, 5, 3, 24), qa, sa)
    assert torch.equal(qa.view(30, 24), steps_of(x.float())[0])
    both = torch.zeros((30, 48), dtype=torch.bfloat16, device="cuda")
    both[:, :24] = x
    q, scale = gdws.empty_rows8(30, 24)
    gdws.norm_quantize_rows(both[:, :24], q, scale, total=both[:, 24:])
    assert torch.equal(both[:, 24:], x) and torch.equal(q, qa.view(30, 24))


def test_binding_says_what_is_wrong():
    x = values(4, 64, "bf16", 1)
    q, scale = gdws.empty_rows8(4, 64)
    y = torch.empty((4, 64), device="cuda")
    cpu = torch.zeros((4, 64))
    for error, run in [(ValueError, lambda: gdws.quantize_rows(cpu, q, scale)), (ValueError, lambda: gdws.quantize_rows(x, q.cpu(), scale)), (ValueError, lambda: gdws.quantize_rows(x, q, scale.cpu())),
                       (TypeError, lambda: gdws.quantize_rows(x.half(), q, scale)), (TypeError, lambda: gdws.quantize_rows(x, q.to(torch.uint8), scale)), (TypeError, lambda: gdws.quantize_rows(x, q, scale.double())),
                       (ValueError, lambda: gdws.quantize_rows(x, q, scale[:3])), (ValueError, lambda: gdws.quantize_rows(x, q, torch.zeros(8, device="cuda")[::2])), (ValueError, lambda: gdws.quantize_rows(x.t(), q, scale)),
                       (gdws.GdwsError, lambda: gdws.quantize_rows(x[:, :60], q, scale)), (gdws.GdwsError, lambda: gdws.quantize_rows(x.expand(4, 64)[:1].expand(4, 64), q, scale)),
                       (ValueError, lambda: gdws.norm_quantize_rows(x, q, scale, weight=torch.ones(63, device="cuda"))), (TypeError, lambda: gdws.norm_quantize_rows(x, q, scale, weight=torch.ones(64, device="cuda").half())),
                       (gdws.GdwsError, lambda: gdws.norm_quantize_rows(x, q, scale, residual=x.float())), (gdws.GdwsError, lambda: gdws.norm_quantize_rows(x, q, scale, eps=0.0)),
                       (gdws.GdwsError, lambda: gdws.dequantize_rows(q, scale, y[:3])), (ValueError, lambda: gdws.pointwise8(q, scale, q, scale, torch.empty((4, 4), device="cuda"), bias=torch.zeros(5, device="cuda")))]:
        with pytest.raises(error):
            run()
    gdws.norm_quantize_rows(x, q, scale, eps=1)          # any number will do


FIRST_CALL = """
import torch
from paper_2110_14871_b200 import gdws
x = torch.arange(64 * 520, device="cuda").remainder(97).float().view(64, 520)
q, scale = gdws.empty_rows8(64, 520)
y, z = torch.empty((64, 64), device="cuda"), torch.empty((64, 520), dtype=torch.bfloat16, device="cuda")
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    gdws.norm_quantize_rows(x, q, scale)
    gdws.pointwise8(q, scale, q, scale, y)
    gdws.dequantize_rows(q, scale, z)
g.replay()
torch.cuda.synchronize()
gdws.rows_status()
v = q.double() * scale.double()[:, None]
assert (y.double() - v @ v.t()).abs().max() < 1e-4 * y.abs().max() and q.any()
print("ok")
"""


def test_the_first_call_of_a_process_may_be_captured():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", FIRST_CALL], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout == "ok\n", r.stderr[-2000:]


def test_streams_graphs_and_the_same_result_twice():
    x, r = values(50, 1000, "bf16", 21), values(50, 1000, "bf16", 22)
    q, scale = gdws.empty_rows8(50, 1000)
    total, y = torch.empty_like(x), torch.empty_like(x)

    def step():
        gdws.norm_quantize_rows(x, q, scale, residual=r, total=total)
        gdws.dequantize_rows(q, scale, y)

    step()
    want = [t.clone() for t in (q, scale, total, y)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y.zero_()
        step()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip((q, scale, total, y), want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for t in (q, scale, total, y):
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((q, scale, total, y), want))
    assert HALF[torch.float32] == torch.finfo(torch.float32).eps / 2

"""gdws_pointwise8 against the product in 64 bits: integer sums are exact, what follows rounds as the interface says; nothing is
written beside y."""
import threading

import numpy as np
import pytest
import torch

from paper_2110_14871_b200 import build as gbuild
from paper_2110_14871_b200 import gdws
from paper_2110_14871_b200 import inputs as gi

from rows8_util import HALF, Field, product_of, steps_of
from util import make_plan, small_spec, to_device

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module", autouse=True)
def built():
    gbuild.build_library()


def rows8(rows, cols, seed, ld=None, shift=0, full=False):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    f = Field(rows, cols, torch.int8, ld, shift)
    f.t.copy_(torch.randint(-128, 128, (rows, cols), generator=gen, device="cuda") if not full else torch.full((rows, cols), -128, device="cuda"))
    return f, torch.rand(rows, generator=gen, device="cuda") * 0.02 + 1e-4


def ceil16(n):
    return (n + 15) // 16 * 16


def compare(rows, K, D, out="bf16", bias=True, relu=False, ldx=None, ldw=None, shift=0, ygap=0, yshift=0, seed=1, full=False):
    x, xs = rows8(rows, K, seed, ldx or ceil16(K), shift, full)
    w, ws = rows8(D, K, seed + 1, ldw or ceil16(K), shift, full)
    b = torch.randn(D, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)) if bias else None
    y = Field(rows, D, TYPES[out], D + ygap, yshift)
    y.t.fill_(float("nan"))
    gdws.pointwise8(x.t, xs, w.t, ws, y.t, bias=b, relu=relu)
    torch.cuda.synchronize()
    gdws.rows_status()
    want, bound = product_of(x.t, xs, w.t, ws, b, relu)
    if out == "bf16":
        bound = bound + HALF[torch.bfloat16] * (want.abs() + bound)
    assert ((y.t.double() - want).abs() <= bound).all(), (rows, K, D)
    for f, name in ((x, "x"), (w, "w"), (y, "y")):
        f.check(name)
    return y.t


@pytest.mark.parametrize("out,relu,bias", [("bf16", False, True), ("f32", True, False)])
@pytest.mark.parametrize("rows,K,D", [(1, 1, 1), (1, 16, 16), (1, 4096, 512), (2, 127, 129), (3, 128, 128), (7, 2049, 300), (16, 1000, 257), (17, 64, 64), (33, 513, 77), (64, 1280, 256),
                                      (65, 33, 1000), (100, 3328, 512), (127, 129, 127), (128, 256, 384), (129, 4097, 65), (200, 300, 400), (257, 640, 255), (300, 17, 513), (513, 1337, 260), (1000, 512, 1000),
                                      (2000, 128, 24), (5000, 48, 300), (20, 2048, 5000), (1, 131071, 3), (1, 300, 70001), (70001, 40, 5)])
def test_sizes(rows, K, D, out, relu, bias):
    compare(rows, K, D, out, bias, relu, seed=rows + K + D)


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("rows,K,D,kernel", [(4100, 300, 2301, gdws.KERNEL8_PAIRS), (2561, 1000, 2600, gdws.KERNEL8_PAIRS), (9000, 100, 1030, gdws.KERNEL8_PAIRS), (300, 5000, 5001, gdws.KERNEL8_SLICES),
                                             (20, 131071, 300, gdws.KERNEL8_SLICES), (40, 3000, 2000, gdws.KERNEL8_SLICES), (100, 8000, 500, gdws.KERNEL8_SLICES), (500, 640, 700, gdws.KERNEL8_SLICES),
                                             (6, 5000, 130, gdws.KERNEL8_FEW), (3, 70000, 9, gdws.KERNEL8_FEW), (1, 200, 20001, gdws.KERNEL8_SLICES)])
def test_every_kernel(rows, K, D, kernel, out):
    """Several tiles for each pair of SMs, rings that go round, clusters of every size, warps that share columns."""
    y = compare(rows, K, D, out, True, True, seed=rows)
    x, xs = rows8(rows, K, 1, ceil16(K))
    w, ws = rows8(D, K, 2, ceil16(K))
    assert kernel == gdws.pointwise8_kernel(x.t, xs, w.t, ws, y)


@pytest.mark.parametrize("rows,K,D,ldx,ldw,shift", [(5, 1337, 70, 1337, 1337, 0), (70, 100, 130, 100, 112, 0), (70, 100, 130, 112, 101, 0), (40, 96, 50, 96, 96, 4), (3, 64, 64, 64, 64, 1), (150, 515, 90, 516, 516, 0)])
def test_any_alignment(rows, K, D, ldx, ldw, shift):
    compare(rows, K, D, "f32", True, False, ldx, ldw, shift)


@pytest.mark.parametrize("rows,K,D", [(1, 512, 200), (40, 512, 200), (300, 200, 300)])
def test_strides_of_every_matrix(rows, K, D):
    compare(rows, K, D, "bf16", True, True, ldx=ceil16(K) + 64, ldw=ceil16(K) + 16, ygap=3, yshift=1)
    compare(rows, K, D, "f32", True, True, ldx=ceil16(K) + 16, ldw=ceil16(K) + 128, ygap=1, yshift=1)


@pytest.mark.parametrize("rows", [1, 20, 300])
def test_largest_sums_are_exact(rows):
    """131071 products of (-128)^2 sum to 2^31 - 2^14; 2^31 - 2^14 is a number of fp32."""
    x, w = (rows8(n, 131071, 1, ceil16(131071), full=True)[0] for n in (rows, 5))
    y = torch.empty((rows, 5), device="cuda")
    one = torch.ones(max(rows, 5), device="cuda")
    gdws.pointwise8(x.t, one[:rows], w.t, one[:5], y)
    assert (y.double() == 131071 * 2.0 ** 14).all()
    with pytest.raises(gdws.GdwsError) as e:
        gdws.pointwise8(*gdws.empty_rows8(1, 131072), *gdws.empty_rows8(5, 131072), y[:1])
    assert e.value.status == gdws.ERR_UNSUPPORTED


@pytest.mark.parametrize("rows,D", [(1, 40), (40, 200), (600, 300)])
def test_not_finite_scales_and_relu(rows, D):
    x, xs = rows8(rows, 256, 3)
    w, ws = rows8(D, 256, 4)
    x.t[0] = 0
    xs[0] = float("nan")
    ws[D // 2] = float("nan")
    for relu in (False, True):
        y = torch.empty((rows, D), device="cuda")
        gdws.pointwise8(x.t, xs, w.t, ws, y, relu=relu)
        nan = torch.zeros((rows, D), dtype=torch.bool, device="cuda")
        nan[0] = True
        nan[:, D // 2] = True
        assert torch.equal(torch.isnan(y), nan)
        assert not relu or (y[~nan] >= 0).all()


def test_no_rows():
    w, ws = rows8(8, 32, 1)
    q, s = gdws.empty_rows8(0, 32)
    gdws.pointwise8(q, s, w.t, ws, torch.empty((0, 8), device="cuda"))


@pytest.mark.parametrize("rows,K,D", [(1, 4096, 600), (50, 700, 300), (700, 512, 520)])
def test_same_bits_on_every_call_stream_and_replay(rows, K, D):
    """Integer sums do not depend on their order: every call gives the same bits; graphs share nothing."""
    want = compare(rows, K, D, "f32").clone()
    x, xs = rows8(rows, K, 1, ceil16(K))
    w, ws = rows8(D, K, 2, ceil16(K))
    b = torch.randn(D, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    ys = [torch.empty((rows, D), device="cuda") for _ in range(4)]
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for g, y in zip(graphs, ys):
        with torch.cuda.graph(g):
            gdws.pointwise8(x.t, xs, w.t, ws, y, bias=b)
    streams = [torch.cuda.Stream() for _ in range(4)]
    torch.cuda.synchronize()
    for s, run in zip(streams, [graphs[0].replay, graphs[1].replay, lambda: gdws.pointwise8(x.t, xs, w.t, ws, ys[2], bias=b), lambda: gdws.pointwise8(x.t, xs, w.t, ws, ys[3], bias=b)]):
        with torch.cuda.stream(s):
            for _ in range(5):
                run()
    torch.cuda.synchronize()
    assert all(torch.equal(y, want) for y in ys)


def test_two_host_threads():
    jobs = [(rows8(r, 512, r, 512), rows8(256, 512, r + 1, 512), torch.empty((r, 256), device="cuda")) for r in (1, 40, 300, 77)]
    torch.cuda.synchronize()

    def work(job):
        (x, xs), (w, ws), y = job
        for _ in range(200):
            gdws.pointwise8(x.t, xs, w.t, ws, y)

    threads = [threading.Thread(target=work, args=(j,)) for j in jobs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    for (x, xs), (w, ws), y in jobs:
        want, bound = product_of(x.t, xs, w.t, ws, None, False)
        assert ((y.double() - want).abs() <= bound).all()


def test_pointwise_stage_of_a_layer_in_8_bits():
    """Depthwise stage in bf16, its rows and the pointwise weights to 8 bits, the product: each step against its definition on what
    the step before left, and the whole within what 8 bits amount to."""
    data = gi.make_layer(small_spec("t", 6, 40, 72, 11, 9, dtype="bf16", seed=5))
    s = data.spec
    plan = make_plan(data)
    G, Gp, _, _ = plan.info()
    x, dw, pw = (to_device(a, "bf16") for a in (data.x, data.dw_w, data.pw_w))
    bias = torch.from_numpy(data.bias).cuda()
    plan.pack_weights(dw, pw, bias)
    pixels = s.N * s.Ho * s.Wo
    z = torch.empty((pixels, Gp), dtype=torch.bfloat16, device="cuda")
    plan.depthwise(x, z, "NHWC")
    q, scale = gdws.empty_rows8(pixels, G)
    w, w_scale = gdws.empty_rows8(s.D, G)
    gdws.quantize_rows(pw, w, w_scale)
    gdws.quantize_rows(z[:, :G], q, scale)
    y = torch.empty((s.N, s.Ho, s.Wo, s.D), dtype=torch.bfloat16, device="cuda")
    gdws.pointwise8(q, scale, w, w_scale, y, bias=bias, relu=True)
    full = torch.empty_like(y)
    plan.set_option(gdws.OPT_RELU, 1)
    plan.pointwise(z, full, "NHWC")
    torch.cuda.synchronize()
    gdws.rows_status()
    qz, sz = steps_of(z[:, :G].float())
    qw, sw = steps_of(pw.float())
    assert torch.equal(q, qz) and torch.equal(scale, sz) and torch.equal(w, qw) and torch.equal(w_scale, sw)
    want, bound = product_of(qz, sz, qw, sw, bias, True)
    assert ((y.view(pixels, s.D).double() - want).abs() <= bound + HALF[torch.bfloat16] * (want.abs() + bound)).all()
    # half a step of either factor times the other, for each product; both results are rounded to bf16, z is what it is
    err = (sz.double()[:, None] / 2) * pw.double().abs().sum(1) + (z[:, :G].double().abs().sum(1) + G * sz.double() / 2)[:, None] * sw.double() / 2
    slack = 2.1 * HALF[torch.bfloat16] * (full.view(pixels, s.D).double().abs() + err) + 1e-5
    assert ((y.view(pixels, s.D).double() - full.view(pixels, s.D).double()).abs() <= err + slack).all()
    plan.destroy()


@pytest.mark.parametrize("rows", [1, 60, 400])
def test_block_of_the_operators(rows):
    """Norm, product with ReLU, 8 bits, product, twice in a row with the residual carried on: as a network's blocks would use them."""
    C, hidden, eps = 320, 1280, 1e-6
    gen = torch.Generator(device="cuda").manual_seed(rows)
    stream = torch.randn((rows, C), generator=gen, device="cuda").to(torch.bfloat16)
    x = torch.randn((rows, C), generator=gen, device="cuda").to(torch.bfloat16)
    for _ in range(2):
        gain = 1 + 0.1 * torch.randn(C, generator=gen, device="cuda")
        weights = []
        for d, k in ((hidden, C), (C, hidden)):
            q, s = gdws.empty_rows8(d, k)
            gdws.quantize_rows(torch.randn((d, k), generator=gen, device="cuda") / np.sqrt(k), q, s)
            weights.append((q, s))
        q, s = gdws.empty_rows8(rows, C)
        h = x.float() + stream.float()
        gdws.norm_quantize_rows(x, q, s, weight=gain, eps=eps, residual=stream, total=stream)
        assert torch.equal(stream, h.to(torch.bfloat16)) and torch.equal(q, steps_of(h * gain)[0])
        a = torch.empty((rows, hidden), dtype=torch.bfloat16, device="cuda")
        gdws.pointwise8(q, s, *weights[0], a, relu=True)
        want, bound = product_of(q, s, *weights[0], None, True)
        assert ((a.double() - want).abs() <= bound + HALF[torch.bfloat16] * (want.abs() + bound)).all()
        hq, hs = gdws.empty_rows8(rows, hidden)
        gdws.quantize_rows(a, hq, hs)
        assert torch.equal(hq, steps_of(a.float())[0])
        x = torch.empty((rows, C), dtype=torch.bfloat16, device="cuda")
        gdws.pointwise8(hq, hs, *weights[1], x)
        want, bound = product_of(hq, hs, *weights[1], None, False)
        assert ((x.double() - want).abs() <= bound + HALF[torch.bfloat16] * (want.abs() + bound)).all()
    gdws.rows_status()

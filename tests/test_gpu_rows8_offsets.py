"""Calls on rows whose operands pass 2^31 elements or bytes: rows at the start, around the border and at the end, against the definitions."""
import pytest
import torch

from paper_2110_14871_b200 import build as gbuild
from paper_2110_14871_b200 import gdws

from rows8_util import HALF, product_of, steps_of
from test_gpu_rows8 import TYPES, norm_bound

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    gbuild.build_library()
    yield
    torch.cuda.empty_cache()


def some_rows(rows, ld):
    """The first and last rows, and those around every 2^31 elements."""
    picks = {0, 1, rows - 2, rows - 1}
    for border in range(1 << 31, rows * ld, 1 << 31):
        picks |= {r for r in range(border // ld - 1, border // ld + 2) if 0 <= r < rows}
    return torch.tensor(sorted(picks), device="cuda")


def fill(t, seed):
    """Values in place, by blocks of rows; a row's first two tell rows apart."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rows, cols = t.shape
    one = torch.randn((1, cols), generator=gen, device="cuda")
    for r in range(0, rows, 1 << 16):
        n = min(1 << 16, rows - r)
        t[r:r + n] = one.to(t.dtype)
        i = torch.arange(r, r + n, device="cuda")
        t[r:r + n, 0] = (i % 251).to(t.dtype) / 64
        t[r:r + n, 1] = (i // 251 % 251).to(t.dtype) / 64


@pytest.mark.parametrize("rows,cols", [(1100000, 2048), (1700001, 1281), (33000, 65553)])
def test_rows(rows, cols):
    x, q, scale = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda"), torch.empty((rows, cols), dtype=torch.int8, device="cuda"), torch.empty(rows, device="cuda")
    fill(x, 1)
    pick = some_rows(rows, cols)
    gdws.quantize_rows(x, q, scale)
    want, want_scale = steps_of(x[pick].float())
    assert torch.equal(q[pick], want) and torch.equal(scale[pick], want_scale)
    y = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda")
    gdws.dequantize_rows(q, scale, y)
    assert torch.equal(y[pick], (want.float() * want_scale[:, None]).bfloat16())
    w = 1 + 0.2 * torch.randn(cols, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda")
    h = x[pick].float() + y[pick].float()
    gdws.norm_quantize_rows(x, q, scale, weight=w, residual=y, total=y)
    assert torch.equal(q[pick], steps_of(h * w)[0]) and torch.equal(y[pick], h.bfloat16())
    want_scale = (h * w).double().abs().amax(1) / 127 / torch.sqrt(h.double().square().mean(1) + 1e-6)
    assert ((scale[pick].double() - want_scale).abs() <= norm_bound(cols) * want_scale).all()


@pytest.mark.parametrize("rows,K,D,ldx,ldw,ldy,out,kernel", [
    (1100000, 2048, 2056, 2048, 2048, 2056, "bf16", gdws.KERNEL8_PAIRS),          # x and y
    (1100000, 1999, 24, 1999, 1999, 24, "f32", gdws.KERNEL8_ANY),                 # x
    (300, 64, 520, 64, 64, 1 << 25, "bf16", gdws.KERNEL8_SLICES),                  # y, far apart
    (1, 4096, 600000, 4096, 4096, 600000, "bf16", gdws.KERNEL8_FEW), (7, 4095, 600000, 4095, 4095, 600000, "f32", gdws.KERNEL8_FEW), (40, 4096, 600000, 4096, 4096, 600000, "bf16", gdws.KERNEL8_PAIRS),      # w
    (5, 512, 72, 1 << 30, 1 << 26, 72, "f32", gdws.KERNEL8_FEW), (70, 512, 72, 1 << 26, (1 << 26) + 1, 72, "f32", gdws.KERNEL8_ANY)])                     # x and w, far apart
def test_products(rows, K, D, ldx, ldw, ldy, out, kernel):
    def matrix(n, cols, ld, dtype):
        return torch.empty((n - 1) * ld + cols, dtype=dtype, device="cuda").as_strided((n, cols), (ld, 1))

    gen = torch.Generator(device="cuda").manual_seed(rows)
    x, w, y = matrix(rows, K, ldx, torch.int8), matrix(D, K, ldw, torch.int8), matrix(rows, D, ldy, TYPES[out])
    for t in (x, w):
        n = t.shape[0]
        one = torch.randint(-128, 128, (min(n, 509), K), generator=gen, device="cuda").to(torch.int8)
        for r in range(0, n, 509):
            t[r:r + 509] = one[:min(509, n - r)]
    xs, ws = torch.rand(rows, generator=gen, device="cuda") * 0.02 + 1e-4, torch.rand(D, generator=gen, device="cuda") * 0.02 + 1e-4
    bias = torch.randn(D, generator=gen, device="cuda")
    assert gdws.pointwise8_kernel(x, xs, w, ws, y) == kernel
    gdws.pointwise8(x, xs, w, ws, y, bias=bias)
    gdws.rows_status()
    pr = torch.cat([some_rows(rows, ldx), some_rows(rows, ldy)]) if rows > 1000 else torch.arange(rows, device="cuda")
    pd = some_rows(D, ldw) if D > 10000 else torch.arange(D, device="cuda")
    want, bound = product_of(x[pr], xs[pr], w[pd], ws[pd], bias[pd], False)
    if out == "bf16":
        bound = bound + HALF[torch.bfloat16] * (want.abs() + bound)
    assert ((y[pr][:, pd].double() - want).abs() <= bound).all()

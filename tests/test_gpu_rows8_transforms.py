"""Tensors of torch's functional transforms have the ordinary type and no memory of their own: the calls on rows refuse them with an
exception.  In a process of its own, which an exception thrown through the interpreter would end."""
import os
import subprocess
import sys

import pytest

from paper_2110_14871_b200 import build as gbuild

pytestmark = pytest.mark.gpu

PROGRAM = """
import torch
from paper_2110_14871_b200 import gdws

rows, k, d = 4, 64, 16
def new():
    q, scale = gdws.empty_rows8(rows, k)
    w, w_scale = gdws.empty_rows8(d, k)
    for t in (q, scale, w, w_scale):
        t.fill_(1)
    x = torch.randn((rows, k), device="cuda")
    return dict(x=x, q=q, scale=scale, residual=torch.randn_like(x), total=torch.empty_like(x), weight=torch.ones(k, device="cuda"), w=w, w_scale=w_scale,
                y=torch.empty((rows, d), device="cuda"), bias=torch.zeros(d, device="cuda"))

CALLS = {
    "quantize": (lambda a: gdws.quantize_rows(a["x"], a["q"], a["scale"]), ("x", "q", "scale")),
    "norm": (lambda a: gdws.norm_quantize_rows(a["x"], a["q"], a["scale"], weight=a["weight"], residual=a["residual"], total=a["total"]), ("x", "q", "scale", "weight", "residual", "total")),
    "dequantize": (lambda a: gdws.dequantize_rows(a["q"], a["scale"], a["x"]), ("q", "scale", "x")),
    "product": (lambda a: gdws.pointwise8(a["q"], a["scale"], a["w"], a["w_scale"], a["y"], bias=a["bias"]), ("q", "scale", "w", "w_scale", "y", "bias")),
}
refused = 0
for name, (call, operands) in CALLS.items():
    call(new())
    for which in operands:
        def run(t):
            call(dict(new(), **{which: t}))
            return t.float().sum()
        t = new()[which]
        transforms = [lambda: torch.func.vmap(run)(torch.stack([t, t]))]
        if t.dtype.is_floating_point:
            transforms += [lambda: torch.func.grad(run)(t), lambda: torch.func.vmap(torch.func.grad(run))(torch.stack([t, t]))]
        for transform in transforms:
            try:
                transform()
            except (RuntimeError, ValueError, TypeError) as e:
                refused += 1
            else:
                print("taken:", name, which)
    call(new())
torch.cuda.synchronize()
gdws.rows_status()
print(refused)
"""


def test_transformed_tensors_are_refused():
    gbuild.build_library()
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", PROGRAM], cwd=root, capture_output=True, text=True, timeout=300)
    # 18 operands, 13 of them floating-point: one transform for each and two more for those
    assert r.returncode == 0 and r.stdout == "44\n", (r.returncode, r.stdout, r.stderr[-2000:])

"""Definitions of the 8-bit row operators in 64 bits, and matrices with guarded surroundings, for the tests of those calls."""
import torch

HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}      # what a rounding to the type errs by, relative to the value


def steps_of(u):
    """(q, scale) of fp32 rows u.  127 u is exact in 64 bits, and the quotient's one rounding there cannot cross the middle of two
    integers: it is at least 2^-25 of itself away from it or exactly on it."""
    u = u.double()
    most = u.abs().amax(1, keepdim=True)
    q = torch.where(most > 0, torch.round(127 * u / torch.where(most > 0, most, 1.0)), torch.zeros_like(u))
    fine = torch.isfinite(u).all(1)
    q[~fine] = 0
    scale = (most[:, 0] / 127).float()
    scale[~fine] = float("nan")
    return q.to(torch.int8), scale


def product_of(q, scale, w, w_scale, bias, relu):
    """(y, bound): the product in 64 bits and how far fp32 arithmetic after the exact sum may be off: the sum's conversion, its
    product with w_scale, and the fused multiply-add round by 2^-24 each."""
    p = (q.double() @ w.double().t()) * w_scale.double() * scale.double()[:, None]
    y = p if bias is None else p + bias.double()
    bound = 2.01 * 2.0 ** -24 * p.abs() + 2.0 ** -24 * y.abs() * 1.01
    return (torch.where(y < 0, torch.zeros_like(y), y) if relu else y), bound


class Field:
    """A matrix [rows][cols] with rows `ld` elements apart inside a larger buffer of a fixed pattern; `shift` elements behind an
    aligned address.  check() fails if anything but the matrix's elements was written."""

    def __init__(self, rows, cols, dtype, ld=None, shift=0):
        ld = cols if ld is None else ld
        size = torch.empty((), dtype=dtype).element_size()
        lead = 256 // size + shift
        n = lead + max(rows - 1, 0) * ld + cols + 256
        self.raw = torch.full((n * size,), 0x5A, dtype=torch.uint8, device="cuda")
        self.flat = self.raw.view(dtype)
        self.t = self.flat.as_strided((rows, cols), (ld, 1), lead)
        inside = torch.zeros(n, dtype=torch.bool, device="cuda")
        inside.as_strided((rows, cols), (ld, 1), lead).fill_(True)
        self.outside = (~inside).repeat_interleave(size)

    def check(self, what):
        assert bool((self.raw[self.outside] == 0x5A).all()), f"bytes around {what} were overwritten"

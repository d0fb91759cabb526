"""The 8-bit row operators: rows of activations to 8-bit integers with a scale each, and the pointwise product that reads them.

A row is what the pointwise stage sums over: the channels of a pixel of an NHWC map, or the features of a token.  A case is a
dict of plain values; `kind` says which entry points a pass takes:

    norm      gdws.norm_quantize_rows (residual added, root-mean-square norm, 8 bits), then gdws.dequantize_rows of its rows
    quantize  gdws.quantize_rows, then gdws.dequantize_rows
    product   gdws.pointwise8: 8-bit rows times 8-bit weights with a scale for each row and output channel, bias, ReLU
    block     the operators in a row: norm, product with ReLU, quantize, product

`rows` rows of `k` values, `d` output channels; `dtype` is that of the unquantized inputs, `out` that of what is written in 16
or 32 bits.  8-bit rows start at multiples of 16 bytes (`packed`: one right behind the other).
"""
import math

import torch

own = False

EPS = 1e-6


def _case(name, kind, rows, k, d=0, dtype="bf16", out="bf16", residual=True, relu=False, packed=False):
    case = {"kind": kind, "rows": rows, "k": k, "d": d, "dtype": dtype, "out": out, "residual": residual, "relu": relu, "packed": packed}
    return dict(case, name=name) if name else case


def listed():
    return [
        # one token of a serving step: launches and latency
        _case("norm_token", "norm", 1, 4096),
        # the tokens of a prompt, or of a training batch that is only read
        _case("norm_batch", "norm", 8192, 4096),
        # fp32 activations, no residual, sizes off every tile
        _case("norm_odd_f32", "norm", 1023, 1531, dtype="f32", residual=False),
        # the intermediate channels of one small image behind a depthwise stage: odd row length, rows without gaps
        _case("quantize_image", "quantize", 196, 1337, packed=True),
        # the same of a batch of 256 8 x 8 maps
        _case("quantize_pixels", "quantize", 16384, 1280, out="f32"),
        # one token: every weight is read for one row
        _case("product_token", "product", 1, 4096, 4096),
        # a few requests served together, a wide layer
        _case("product_few", "product", 16, 4096, 16384),
        # pointwise stage of a CIFAR layer: many pixels, few output channels
        _case("product_pixels", "product", 16384, 1280, 256, relu=True),
        # odd sizes throughout, fp32 sums kept
        _case("product_ragged", "product", 637, 1203, 1001, out="f32"),
        # a prompt through a wide layer: the most arithmetic
        _case("product_prompt", "product", 8192, 4096, 8192),
        # feed-forward block, one token and a batch of tokens
        _case("block_token", "block", 1, 2048, 8192),
        _case("block_batch", "block", 2048, 2048, 8192),
    ]


def _log(rng, lo, hi):
    return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))


_MOST = {"norm": 3.3e7, "quantize": 2e7}      # elements of a drawn case


def draw(rng):
    kind = rng.choice(["norm", "quantize", "product", "product", "product", "block"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    # behind a norm the values before their rounding to 8 bits are fp32 sums and products themselves: bf16 is what they are good for
    out = rng.choice(["bf16", "bf16", "f32"]) if kind in ("quantize", "product") else "bf16"
    while True:
        if kind in _MOST:
            case = _case(None, kind, _log(rng, 1, 20000), _log(rng, 16, 16384), 0, dtype, out, rng.random() < 0.7, False, rng.random() < 0.2)
            if case["rows"] * case["k"] <= _MOST[kind]:
                return case
            continue
        most = 20000 if kind == "product" else 4096
        rows, k, d = _log(rng, 1, most), _log(rng, 16, most), _log(rng, 16, most)
        if rng.random() < 0.6:
            k, d = max(16, k // 16 * 16), max(16, d // 16 * 16)
        case = _case(None, kind, rows, k, d, dtype, out, True, rng.random() < 0.5, rng.random() < 0.1)
        if 2.0 * rows * k * d <= (4e11 if kind == "product" else 6e10) and max(rows * k, rows * d, k * d) <= 6e7:
            return case


_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _rows8(rows, k, packed):
    """8-bit rows and their scales; rows 16 bytes apart or packed."""
    ld = k if packed else (k + 15) // 16 * 16
    return torch.zeros((rows, ld), dtype=torch.int8, device="cuda")[:, :k], torch.zeros(rows, dtype=torch.float32, device="cuda")


def _weights8(gen, d, k, packed):
    """Weights of a trained layer in 8 bits, a scale for each output channel."""
    w = torch.randn((d, k), generator=gen, device="cuda") / math.sqrt(k)
    q, scale = _rows8(d, k, packed)
    top = w.abs().amax(1)
    q.copy_((w * (127.0 / top)[:, None]).round())
    scale.copy_(top / 127)
    return q, scale


def _activations(gen, rows, k, dtype):
    """Activations: some channels are an order of magnitude larger than the others."""
    x = torch.randn((rows, k), generator=gen, device="cuda")
    x *= torch.where(torch.rand(k, generator=gen, device="cuda") < 0.01, 12.0, 1.0)
    return x.to(_TYPES[dtype])


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rows, k, d, kind, packed = (case[n] for n in ("rows", "k", "d", "kind", "packed"))
    st = dict(case, out_type=_TYPES[case["out"]])
    if kind != "product":
        st["x"] = _activations(gen, rows, k, case["dtype"])
        st["q"], st["scale"] = _rows8(rows, k, packed)
    if kind in ("norm", "block"):
        st["weight"] = 1 + 0.2 * torch.randn(k, generator=gen, device="cuda")
        st["residual"] = (4 * _activations(gen, rows, k, "f32")).to(st["x"].dtype) if case["residual"] else None
        st["total"] = torch.empty_like(st["x"]) if case["residual"] else None
    if kind in ("norm", "quantize"):
        st["values"] = torch.empty((rows, k), dtype=st["out_type"], device="cuda")
    if kind == "product":
        x = _activations(gen, rows, k, "f32")
        st["q"], st["scale"] = _rows8(rows, k, packed)
        top = x.abs().amax(1)
        st["q"].copy_((x * (127.0 / top)[:, None]).round())
        st["scale"].copy_(top / 127)
    if kind in ("product", "block"):
        st["w"], st["w_scale"] = _weights8(gen, d, k, packed)
        st["bias"] = 0.1 * torch.randn(d, generator=gen, device="cuda")
        st["y"] = torch.empty((rows, d), dtype=st["out_type"], device="cuda")
    if kind == "block":
        st["hq"], st["h_scale"] = _rows8(rows, d, packed)
        st["w2"], st["w2_scale"] = _weights8(gen, k, d, packed)
        st["bias2"] = 0.1 * torch.randn(k, generator=gen, device="cuda")
        st["y2"] = torch.empty((rows, k), dtype=st["out_type"], device="cuda")
    return st


# ---- the operators in elementary operations, 32 bits

def _plain_quantize(u):
    """u to integers of at most 127 in magnitude and the scale of each row: q = round(127 u / max |u|), scale = max |u| / 127.
    The quotient in 64 bits: in 32 some of those halfway between two integers fall on the wrong side."""
    top = u.abs().amax(1, keepdim=True)
    steps = 127 * u.double() / torch.where(top > 0, top, 1).double()
    return steps.round().float(), top[:, 0] / 127


def _plain_norm_quantize(x, residual, weight):
    """h = x + residual; the 8 bits are those of h * weight, the norm 1 / sqrt(mean h^2 + eps) goes into the scale."""
    h = x.float() if residual is None else x.float() + residual.float()
    q, scale = _plain_quantize(h * weight)
    return q, scale / (h.square().mean(1) + EPS).sqrt(), h.to(x.dtype)


def _plain_product(q, scale, w, w_scale, bias, relu, out):
    y = (q.float() @ w.float().t()) * w_scale * scale[:, None] + bias
    return (y.clamp_min(0) if relu else y).to(out)


def _plain(st):
    kind, out = st["kind"], st["out_type"]
    if kind == "product":
        return _plain_product(st["q"], st["scale"], st["w"], st["w_scale"], st["bias"], st["relu"], out)
    if kind == "quantize":
        q, scale = _plain_quantize(st["x"].float())
        return {"values": (q * scale[:, None]).to(out), "scale": scale}
    q, scale, total = _plain_norm_quantize(st["x"], st["residual"], st["weight"])
    if kind == "norm":
        return {"values": (q * scale[:, None]).to(out), "scale": scale, "total": total if st["residual"] is not None else None}
    h = _plain_product(q, scale, st["w"], st["w_scale"], st["bias"], True, out)
    hq, h_scale = _plain_quantize(h.float())
    return {"y": _plain_product(hq, h_scale, st["w2"], st["w2_scale"], st["bias2"], False, out), "total": total}


# ---- the framework's calls

def _own(st):
    from paper_2110_14871_b200 import gdws
    kind = st["kind"]
    if kind == "product":
        gdws.pointwise8(st["q"], st["scale"], st["w"], st["w_scale"], st["y"], bias=st["bias"], relu=st["relu"])
        return st["y"]
    if kind == "quantize":
        gdws.quantize_rows(st["x"], st["q"], st["scale"])
        gdws.dequantize_rows(st["q"], st["scale"], st["values"])
        return {"values": st["values"], "scale": st["scale"]}
    gdws.norm_quantize_rows(st["x"], st["q"], st["scale"], weight=st["weight"], eps=EPS, residual=st["residual"], total=st["total"])
    if kind == "norm":
        gdws.dequantize_rows(st["q"], st["scale"], st["values"])
        return {"values": st["values"], "scale": st["scale"], "total": st["total"]}
    gdws.pointwise8(st["q"], st["scale"], st["w"], st["w_scale"], st["y"], bias=st["bias"], relu=True)
    gdws.quantize_rows(st["y"], st["hq"], st["h_scale"])
    gdws.pointwise8(st["hq"], st["h_scale"], st["w2"], st["w2_scale"], st["y2"], bias=st["bias2"])
    return {"y": st["y2"], "total": st["total"]}


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    """Inputs once, outputs once; rows between two operators of a pass (the 8-bit rows, a block's hidden layer) are none of
    them.  Operations: the products' multiply-adds, ten an element for the rest."""
    rows, k, d = case["rows"], case["k"], case["d"]
    size, out = (4 if case[n] == "f32" else 2 for n in ("dtype", "out"))
    if case["kind"] == "product":
        return {"bytes": rows * (k + 4 + d * out) + d * (k + 8), "flops": 2.0 * rows * k * d}
    total = {"bytes": rows * k * size, "flops": 10.0 * rows * k}
    if case["kind"] in ("norm", "block"):
        total["bytes"] += 4 * k + (2 * rows * k * size if case["residual"] else 0)
    if case["kind"] == "block":
        total["bytes"] += 2 * d * k + 8 * (d + k) + rows * k * out
        total["flops"] += 4.0 * rows * k * d
    else:
        total["bytes"] += rows * k * out + 4 * rows
    return total


# ---- the definitions in 64 bits

def _exact_rows(v):
    """(values, scale) of v's rows held in 8 bits."""
    most = torch.max(torch.abs(v), 1).values
    steps = torch.round(v * 127 / most.clamp_min(1e-300)[:, None])
    return steps * (most / 127)[:, None], most / 127


def exact(case, seed):
    st = prepare(case, seed)
    f = {n: v.double() for n, v in st.items() if isinstance(v, torch.Tensor)}
    kind = case["kind"]
    if kind == "product":
        y = torch.matmul(f["q"] * f["scale"][:, None], (f["w"] * f["w_scale"][:, None]).t()) + f["bias"]
        return torch.relu(y) if case["relu"] else y
    if kind == "quantize":
        values, scale = _exact_rows(f["x"])
        return {"values": values, "scale": scale}
    total = f["x"] + f["residual"] if case["residual"] else f["x"]
    normed = total / torch.sqrt((total * total).sum(1, keepdim=True) / case["k"] + EPS) * f["weight"]
    values, scale = _exact_rows(normed)
    total = total if case["residual"] else None
    if kind == "norm":
        return {"values": values, "scale": scale, "total": total}
    hidden = torch.relu(torch.matmul(values, (f["w"] * f["w_scale"][:, None]).t()) + f["bias"])
    hidden = _exact_rows(hidden.to(st["out_type"]).double())[0]      # the hidden layer is a tensor of the output's type
    return {"y": torch.matmul(hidden, (f["w2"] * f["w2_scale"][:, None]).t()) + f["bias2"], "total": total}

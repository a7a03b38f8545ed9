"""The 4-bit operators of the library, each one pass through its public entry points, beside their plain forms.

Four kinds of work, as programs that use the library have them:

  quantize  rows of a map written in 4 bits with block scales (dc_q4_quantize) and read back (dc_q4_dequantize): what is held in
            4 bits is compared as the values that it stands for
  read      a quantised matrix back in bf16 or fp32 (dc_q4_dequantize)
  product   y = act(alpha * X W^T + bias + residual) of two quantised matrices (dc_q4_product): a 1x1 layer or a classifier whose input
            map and weights are both held in 4 bits
  forward   the same from rows in bf16 or fp32, quantised by the call itself (dc_q4_forward)

Formats.  Codes are e2m1 (0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign).  "mx4": blocks of 32 columns share a scale 2^e,
e = floor(log2(largest magnitude)) - 2.  "nv4": blocks of 16 share a scale s in e4m3, s = largest magnitude / (6 g) rounded, and the whole
matrix a power of two g.  Values are rounded to the nearest code, ties to the even one, and cut off at 6.

Shapes are those of 1x1 layers of the network in paper_2301_12187_b200/inputs.py, and generic ones up to 16384 rows and 8192 columns.
"""
import math

import torch

own = False                                      # whether run() makes the library's calls; set from outside

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BLOCK = {"mx4": 32, "nv4": 16}
BYTES_MAX, FLOPS_MAX = 6.5e8, 1.2e12             # bounds on one drawn case: below the largest listed ones


# --------------------------------------------------------------------------- the cases


def listed():
    return [
        # One token's activations, written in 4 bits on their own: latency.
        dict(name="quantize_token", kind="quantize", fmt="nv4", rows=1, cols=4096, dtype="bf16", relu=False),
        # A hidden map of the network between two 1x1 layers: 128 images of 28 x 28, 192 channels behind a ReLU6.
        dict(name="quantize_map28", kind="quantize", fmt="mx4", rows=128 * 28 * 28, cols=192, dtype="bf16", relu=True),
        # The activations of a long batch of tokens: bound by memory.
        dict(name="quantize_wide", kind="quantize", fmt="nv4", rows=16384, cols=8192, dtype="bf16", relu=False),
        # Odd rows and columns in fp32: every row begins unaligned and ends inside a block.
        dict(name="quantize_ragged", kind="quantize", fmt="mx4", rows=5001, cols=1003, dtype="f32", relu=False),
        # A layer's 4-bit weights read back in bf16.
        dict(name="read_weights", kind="read", fmt="nv4", rows=8192, cols=8192, dtype="bf16", relu=False),
        # A small odd matrix read back in fp32.
        dict(name="read_ragged", kind="read", fmt="mx4", rows=777, cols=1003, dtype="f32", relu=False),
        # The network's head: 1x1, 320 -> 1280 at 7 x 7 on 128 images, ReLU6.
        dict(name="product_head", kind="product", fmt="mx4", rows=128 * 7 * 7, c_in=320, c_out=1280, dtype="bf16", bias=True,
             residual=False, act=1),
        # A large square product: bound by the tensor core.
        dict(name="product_large", kind="product", fmt="nv4", rows=8192, c_in=8192, c_out=8192, dtype="bf16", bias=False,
             residual=False, act=0),
        # Odd sizes, fp32 results with bias and residual: logits of a classifier.
        dict(name="product_ragged", kind="product", fmt="nv4", rows=1001, c_in=1000, c_out=1003, dtype="f32", bias=True,
             residual=True, act=0),
        # One token through a linear layer: the weights are read once, latency.
        dict(name="forward_token", kind="forward", fmt="nv4", rows=1, c_in=4096, c_out=4096, dtype="bf16", bias=True,
             residual=False, act=0),
        # Sixteen tokens at once through a wider layer, added to what went around it.
        dict(name="forward_tokens16", kind="forward", fmt="mx4", rows=16, c_in=8192, c_out=8192, dtype="bf16", bias=True,
             residual=True, act=0),
        # The expansion of an inverted-residual block: 24 -> 144 at 56 x 56 on 64 images, ReLU6; bound by writing the result.
        dict(name="forward_expand56", kind="forward", fmt="mx4", rows=64 * 56 * 56, c_in=24, c_out=144, dtype="bf16", bias=True,
             residual=False, act=1),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    """Mostly multiples of 8, as layers have them; one in four is any number."""
    v = _log_int(rng, lo, hi)
    return v if rng.random() < 0.25 else min(hi, max(8, v // 8 * 8))


def draw(rng):
    kind = rng.choice(["quantize", "quantize", "read", "product", "product", "product", "forward", "forward", "forward"])
    fmt = rng.choice(["mx4", "nv4"])
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    if kind in ("quantize", "read"):
        case = dict(kind=kind, fmt=fmt, rows=_log_int(rng, 1, 200000), cols=_width(rng, 16, 8192), dtype=dtype,
                    relu=kind == "quantize" and rng.random() < 0.3)
    else:
        rows = _log_int(rng, 1, 64) if kind == "forward" and rng.random() < 0.5 else _log_int(rng, 1, 200000)
        case = dict(kind=kind, fmt=fmt, rows=rows, c_in=_width(rng, 16, 8192), c_out=_width(rng, 8, 8192), dtype=dtype,
                    bias=rng.random() < 0.7, residual=rng.random() < 0.3, act=rng.randint(0, 1))
    while True:
        w = work(case)
        over = max(w["bytes"] / BYTES_MAX, w["flops"] / FLOPS_MAX)
        if over <= 1.0 or case["rows"] == 1:
            return case
        case["rows"] = max(1, int(case["rows"] / max(over, 1.01)))


def _elem(case):
    return 2 if case["dtype"] == "bf16" else 4


def _q4_bytes(rows, cols, fmt):
    return rows * cols * 0.5 + rows * -(-cols // BLOCK[fmt])


def work(case):
    e, rows = _elem(case), case["rows"]
    if case["kind"] in ("quantize", "read"):
        cols = case["cols"]
        q = _q4_bytes(rows, cols, case["fmt"])
        whole = rows * cols * e
        # written in 4 bits, and read back from them
        return {"bytes": 2 * whole + 2 * q if case["kind"] == "quantize" else whole + q, "flops": 2.0 * rows * cols}
    c_in, c_out = case["c_in"], case["c_out"]
    x = _q4_bytes(rows, c_in, case["fmt"]) if case["kind"] == "product" else rows * c_in * e
    y = rows * c_out * e
    return {"bytes": x + _q4_bytes(c_out, c_in, case["fmt"]) + (2 if case["residual"] else 1) * y + (4 * c_out if case["bias"] else 0),
            "flops": 2.0 * rows * c_in * c_out}


# --------------------------------------------------------------------------- inputs


def _raw(case, seed):
    """Inputs in full precision: activations with channels of different size, weights of a layer's fan-in."""
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 7919 + 17)
    rows, dtype = case["rows"], DTYPES[case["dtype"]]
    cols = case["cols"] if "cols" in case else case["c_in"]
    gain = torch.exp(0.5 * torch.randn(cols, generator=g, device="cuda"))
    x = torch.randn(rows, cols, generator=g, device="cuda") * gain
    if case.get("relu"):
        x = x.clamp(0.0, 6.0)
    raw = {"x": x.to(dtype)}
    if "c_out" in case:
        raw["w"] = torch.randn(case["c_out"], cols, generator=g, device="cuda") / math.sqrt(cols)
        raw["bias"] = torch.randn(case["c_out"], generator=g, device="cuda") * 0.1 if case["bias"] else None
        raw["residual"] = torch.randn(rows, case["c_out"], generator=g, device="cuda").to(dtype) if case["residual"] else None
    return raw


def _tensor_scale(t, fmt):
    """nv4: the smallest power of two with which the largest block scale stays in e4m3."""
    if fmt == "mx4":
        return 1.0
    top = float(t.abs().max())
    return 2.0 ** math.ceil(math.log2(top / (6.0 * 448.0))) if top > 0 else 1.0


def prepare(case, seed):
    raw, fmt = _raw(case, seed), case["fmt"]
    s = {"case": case, "fmt": fmt, "g": _tensor_scale(raw["x"], fmt), "x": raw["x"]}
    rows, dtype = case["rows"], DTYPES[case["dtype"]]
    cols = raw["x"].shape[1]
    s["y"] = torch.empty(rows, case.get("c_out", cols), dtype=dtype, device="cuda")
    if "c_out" in case:
        s["gw"] = _tensor_scale(raw["w"], fmt)
        s["w"] = _pack(*_quantize(raw["w"], fmt, s["gw"]))
        s["bias"], s["residual"], s["act"] = raw["bias"], raw["residual"], case["act"]
    if case["kind"] in ("read", "product"):
        s["xq"] = _pack(*_quantize(raw["x"], fmt, s["g"]))
    if own:
        _own_handles(s, raw)
    if case["kind"] in ("read", "product"):
        del s["x"]
    return s


# --------------------------------------------------------------------------- the plain forms


def _pow2(e):
    """2^e in fp32 of whole numbers from -126 to 127."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _floor_log2(v):
    return torch.frexp(v)[1] - 1


def _quantize(x, fmt, g):
    """Codes 0..15 of rows padded to whole blocks, and the scales as values, [rows, blocks]."""
    b = BLOCK[fmt]
    x = torch.nn.functional.pad(x.float(), (0, -x.shape[1] % b)).reshape(x.shape[0], -1, b)
    top = x.abs().amax(-1)
    if fmt == "mx4":
        scale = torch.where(top > 0, _pow2((_floor_log2(top) - 2).clamp(-126, 127)), torch.zeros_like(top))
    else:
        v = (top / (6.0 * g)).clamp(max=448.0)
        step = _pow2(_floor_log2(v).clamp(min=-6) - 3)
        scale = torch.round(v / step) * step * g
    u = torch.where(scale[..., None] > 0, x / scale[..., None], torch.zeros_like(x))
    m = u.abs()
    step = torch.where(m < 2.0, 0.5, torch.where(m < 4.0, 1.0, 2.0))
    m = (torch.round(m / step) * step).clamp(max=6.0)
    code = torch.where(m < 2.0, 2.0 * m, torch.where(m < 4.0, m + 2.0, 0.5 * m + 4.0))
    return (code + torch.where(u < 0, 8.0, 0.0)).to(torch.uint8).reshape(x.shape[0], -1), scale


def _pack(code, scale):
    """Two codes a byte, the first in the low half, and the scales: as a program holds a 4-bit matrix."""
    return code[:, 0::2] | (code[:, 1::2] << 4), scale


def _values(packed, cols):
    """A 4-bit matrix as the fp32 values that it stands for."""
    codes, scale = packed
    code = torch.stack((codes & 15, codes >> 4), -1).reshape(codes.shape[0], -1)
    k = (code & 7).float()
    m = torch.where(k < 4.0, 0.5 * k, torch.where(k < 6.0, k - 2.0, 2.0 * k - 8.0))
    v = torch.where(code > 7, -m, m).reshape(code.shape[0], scale.shape[1], -1) * scale[..., None]
    return v.reshape(code.shape[0], -1)[:, :cols]


def _plain(s):
    case, fmt = s["case"], s["fmt"]
    dtype = DTYPES[case["dtype"]]
    if case["kind"] == "quantize":
        return _values(_pack(*_quantize(s["x"], fmt, s["g"])), case["cols"]).to(dtype)
    if case["kind"] == "read":
        return _values(s["xq"], case["cols"]).to(dtype)
    xq = s["xq"] if case["kind"] == "product" else _pack(*_quantize(s["x"], fmt, s["g"]))
    y = torch.matmul(_values(xq, case["c_in"]), _values(s["w"], case["c_in"]).t())
    if s["bias"] is not None:
        y = y + s["bias"]
    if s["residual"] is not None:
        y = y + s["residual"].float()
    if s["act"]:
        y = y.clamp(0.0, 6.0)
    return y.to(dtype)


# --------------------------------------------------------------------------- the library's calls


def _own_handles(s, raw):
    """What a program keeps: the matrices in the library's 4-bit layout, the buffers of results, and a workspace."""
    from paper_2301_12187_b200 import dc
    case = s["case"]
    code = dc.MX4 if s["fmt"] == "mx4" else dc.NV4
    rows, cols = raw["x"].shape
    s["hx"] = dc.Q4Matrix(rows, cols, code, s["g"]) if case["kind"] != "forward" else None
    if case["kind"] in ("read", "product"):
        dc.q4_quantize(raw["x"], s["hx"])
    if "c_out" in case:
        s["hw"] = dc.Q4Matrix(case["c_out"], cols, code, s["gw"])
        dc.q4_quantize(raw["w"], s["hw"])
        s["ws"] = torch.zeros(dc.q4_workspace_bytes(rows, cols, code), dtype=torch.uint8, device="cuda")


def _own(s):
    from paper_2301_12187_b200 import dc
    kind = s["case"]["kind"]
    if kind == "quantize":
        dc.q4_quantize(s["x"], s["hx"])
        dc.q4_dequantize(s["hx"], s["y"])
    elif kind == "read":
        dc.q4_dequantize(s["hx"], s["y"])
    elif kind == "product":
        dc.q4_product(s["hx"], s["hw"], s["bias"], s["act"], s["residual"], s["y"], s["ws"])
    else:
        dc.q4_forward(s["x"], s["hw"], s["g"], s["bias"], s["act"], s["residual"], s["y"], s["ws"])
    return s["y"]


def run(state):
    return _own(state) if own else _plain(state)


# --------------------------------------------------------------------------- from the definition, in 64 bits

E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _nearest(v, grid):
    """The point of an increasing grid nearest to each v >= 0; between two of them the one at an even place."""
    grid = torch.tensor(grid, dtype=torch.float64, device=v.device)
    mid = (grid[1:] + grid[:-1]) / 2
    low = torch.bucketize(v, mid, right=False)           # borders strictly below v
    high = torch.bucketize(v, mid, right=True)           # borders at or below v
    return grid[torch.where((low != high) & (high % 2 == 0), high, low)]


def _e4m3_grid():
    return [m * 2.0 ** -9 for m in range(8)] + [(8 + m) * 2.0 ** (e - 3) for e in range(-6, 9) for m in range(8) if (e, m) != (8, 7)]


def _stands_for(t, fmt, g):
    """The values that the 4-bit form of t stands for, block by block of the definition."""
    rows, cols = t.shape
    b = BLOCK[fmt]
    out = torch.zeros(rows, -(-cols // b) * b, dtype=torch.float64, device=t.device)
    out[:, :cols] = t.double()
    blocks = out.view(-1, b)
    for at in range(0, blocks.shape[0], 1 << 21):        # in pieces, for the memory of the 64-bit intermediates
        x = blocks[at:at + (1 << 21)]
        top = x.abs().max(dim=1, keepdim=True).values
        if fmt == "mx4":
            # the largest power of two not above the largest magnitude, looked up: a logarithm of 8 may come out below 3
            powers = torch.tensor([2.0 ** e for e in range(-120, 128)], dtype=torch.float64, device=t.device)
            scale = powers[(torch.bucketize(top, powers, right=True) - 1).clamp(min=0)] / 4
        else:
            scale = _nearest((top / (6 * g)).clamp(max=448.0), _e4m3_grid()) * g
        u = torch.where(scale > 0, x.abs() / scale.clamp(min=1e-300), torch.zeros_like(x))
        blocks[at:at + (1 << 21)] = torch.sign(x) * _nearest(u, E2M1) * scale
    return out[:, :cols]


def exact(case, seed):
    raw, fmt = _raw(case, seed), case["fmt"]
    x = _stands_for(raw["x"], fmt, _tensor_scale(raw["x"], fmt))
    if "c_out" not in case:
        return x
    y = x @ _stands_for(raw["w"], fmt, _tensor_scale(raw["w"], fmt)).t()
    if raw["bias"] is not None:
        y = y + raw["bias"].double()
    if raw["residual"] is not None:
        y = y + raw["residual"].double()
    return y.clamp(0, 6) if case["act"] else y

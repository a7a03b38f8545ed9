"""4-bit matrices on the GPU against the oracle in 64 bits.

Quantising and reading back are exact: every byte is compared.  Products of quantised values are exact, their sums are in fp32:
an element may be off by what its sum loses, at most one unit in the last place of the largest partial sum for each of the K additions
(2^-23 K S, S the sum of the products' magnitudes), by two roundings of fp32 behind it (scale and bias, residual), and by the rounding of the
result to its type (finfo.eps / 2 of the value)."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from oracle import q4_oracle as Q
from paper_2301_12187_b200 import dc
from tests.parity_util import Guarded

FMTS = [dc.MX4, dc.NV4]
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def rand(rows, cols, seed, scale=1.0, dtype="f32"):
    r = np.random.default_rng(seed)
    x = (r.standard_normal((rows, cols)) * np.exp(0.7 * r.standard_normal((1, cols))) * scale).astype(np.float32)
    return torch.from_numpy(x).to(TYPES[dtype])


def np64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def matrix(rows, cols, fmt, g=1.0):
    """A Q4Matrix between guards, every byte of it set to a pattern."""
    q = dc.Q4Matrix(rows, cols, fmt, g)
    guard = Guarded(torch, (int(q.layout.bytes),), torch.uint8, fill=0x5A)
    q.data = guard.t
    return q, guard


def check_quantized(x, fmt, g, q, guard):
    torch.cuda.synchronize()
    guard.check("quantised matrix")
    rows, cols = q.rows, q.cols
    code, byte = Q.unpack(q.data.cpu().numpy(), rows, cols, fmt)
    ref_code, ref_byte = Q.quantize(np64(x).reshape(rows, cols), fmt, g)
    nb = ref_byte.shape[1]
    assert (byte[:rows, :nb] == ref_byte).all(), np.argwhere(byte[:rows, :nb] != ref_byte)[:4]
    assert (byte[rows:] == 0).all() and (byte[:rows, nb:] == 0).all()
    have = code[:, :cols]
    same = (have == ref_code) | (ref_code < 0) | ((have & 7 == 0) & (ref_code & 7 == 0))       # a zero's sign is free
    assert same.all(), [(int(r), int(c), int(have[r, c]), int(ref_code[r, c])) for r, c in np.argwhere(~same)[:4]]
    finite = ref_code.min(axis=1) >= 0
    assert (code[finite, cols:] == 0).all()
    return ref_code, ref_byte


SHAPES = [(1, 1), (1, 16), (2, 17), (3, 24), (130, 33), (128, 64), (127, 128), (257, 1003), (5, 4097), (300, 256), (64, 272), (1, 8192)]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_quantize_and_read_back(rows, cols, fmt, dtype):
    x = rand(rows, cols, rows * 31 + cols, dtype=dtype).cuda()
    g = 1.0 if fmt == dc.MX4 else dc.q4_tensor_scale(float(x.float().abs().max()))
    q, guard = matrix(rows, cols, fmt, g)
    dc.q4_quantize(x, q)
    code, byte = check_quantized(x, fmt, g, q, guard)
    for out in TYPES.values():
        y = Guarded(torch, (rows, cols), out, fill=7.0)
        dc.q4_dequantize(q, y.t)
        torch.cuda.synchronize()
        y.check("values")
        assert (np64(y.t) == Q.values(code, byte, fmt, g)).all()


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("cols,stride", [(24, 40), (33, 50), (64, 65), (100, 104)])
def test_strided_rows(cols, stride, fmt, dtype):
    """A slice of channels in, and into a slice of channels: what lies between the rows is neither read nor changed."""
    rows = 150
    wide = torch.full((rows, stride), float("nan"), device="cuda", dtype=TYPES[dtype])
    x = wide[:, :cols]
    x.copy_(rand(rows, cols, cols, dtype=dtype))
    g = 1.0 if fmt == dc.MX4 else 2.0 ** -7
    q, guard = matrix(rows, cols, fmt, g)
    dc.q4_quantize(x, q)
    code, byte = check_quantized(x, fmt, g, q, guard)
    out = torch.full((rows, stride), 3.0, device="cuda", dtype=TYPES[dtype])
    dc.q4_dequantize(q, out[:, :cols])
    assert (np64(out[:, :cols]) == Q.values(code, byte, fmt, g)).all() and (out[:, cols:] == 3.0).all()


@pytest.mark.parametrize("fmt", FMTS)
def test_edges_of_the_formats(fmt):
    """Ties, borders, zeros of both signs, the smallest and the largest numbers, infinities and NaN, scales beyond the format's range."""
    b = Q.block_of(fmt)
    g = 1.0
    rows = []
    ties = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 0.0, -0.0, -0.25, -2.5, 4.999999, 5.000001, 0.24999999, 0.25000003]
    for s in (1.0, 0.5, 2.0 ** -6, 96.0, 448.0):
        rows.append([t * s for t in ties])
    up, down = np.nextafter(np.float32(1), np.float32(2)), np.nextafter(np.float32(1), np.float32(0))
    for s in (1.0, 1.125, 1.25, 1.5, 1.75, 1.875, 0.8125):             # values next to the borders of blocks with that scale
        rows.append([6.0 * s] + [float(np.float32(t * s) * f) for t in (0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0) for f in (up, down)] + [0.0])
    for top in (0.0, 1e-45, 2.0 ** -149 * 3, 1e-38, 2.0 ** -126, 2.0 ** -125, 2.0 ** -124 * 1.99, 3.4e38, 2688.0, 3000.0, 1e30, 6 * 2.0 ** -10, 6.1 * 2.0 ** -10,
                6 * 2.0 ** -9 * 1.5, 8.0, 7.9999995, 4.0):
        rows.append([top, -top / 3, top / 5, -top / 7] + [top * t / 12 for t in range(12)])
    for bad in (np.nan, np.inf, -np.inf):
        rows.append([1.0, bad] + [2.0] * 14)
    x = np.zeros((len(rows), b + 16), dtype=np.float32)
    x[:, :16] = np.array(rows, dtype=np.float32)
    x[:, b:] = 1.0                                                     # the next block is not touched by what this one holds
    for scale in ([1.0] if fmt == dc.MX4 else [1.0, 2.0 ** -9, 2.0 ** 20, 2.0 ** -100, 2.0 ** 100]):
        t = torch.from_numpy(x).cuda()
        q, guard = matrix(len(rows), b + 16, fmt, scale)
        dc.q4_quantize(t, q)
        code, byte = check_quantized(t, fmt, scale, q, guard)
        y = torch.empty_like(t)
        dc.q4_dequantize(q, y)
        odd = (code < 0).any(1)
        have = np64(y)
        assert odd.sum() == 3 and np.isnan(have[odd, :b]).all()
        assert (have[~odd] == Q.values(code[~odd], byte[~odd], fmt, scale)).all()


def bound(xv, wv, scale_s, ref, dtype, k):
    s = np.abs(xv) @ np.abs(wv).T
    eps = torch.finfo(TYPES[dtype]).eps / 2
    return eps * np.abs(ref) + (k + 3) * 2.0 ** -23 * (s + np.abs(scale_s) + np.abs(ref)) + 1e-37


def run_product(rows, c_in, c_out, fmt, dtype, bias, residual, act, forward, seed=0, inplace=False):
    r = np.random.default_rng(seed + rows * 7 + c_in * 3 + c_out)
    x = rand(rows, c_in, seed + 1, dtype=dtype).cuda()
    w = rand(c_out, c_in, seed + 2, 1.0 / np.sqrt(c_in)).cuda()
    gx, gw = (1.0, 1.0) if fmt == dc.MX4 else (dc.q4_tensor_scale(float(x.float().abs().max())), dc.q4_tensor_scale(float(w.abs().max())))
    wq = dc.Q4Matrix(c_out, c_in, fmt, gw)
    dc.q4_quantize(w, wq)
    b = torch.from_numpy(r.standard_normal(c_out).astype(np.float32)).cuda() if bias else None
    res = torch.from_numpy(r.standard_normal((rows, c_out)).astype(np.float32)).to(TYPES[dtype]).cuda() if residual else None
    y = Guarded(torch, (rows, c_out), TYPES[dtype], fill=77.0)
    rin = res
    if inplace:
        y.t.copy_(res)
        rin = y.t
    ws = torch.zeros(dc.q4_workspace_bytes(rows, c_in, fmt), dtype=torch.uint8, device="cuda")
    if forward:
        dc.q4_forward(x, wq, gx, b, act, rin, y.t, ws)
    else:
        xq = dc.Q4Matrix(rows, c_in, fmt, gx)
        dc.q4_quantize(x, xq)
        dc.q4_product(xq, wq, b, act, rin, y.t, ws)
    assert dc.workspace_status(ws) == dc.OK
    y.check("result")
    xv, wv = Q.stands_for(np64(x), fmt, gx), Q.stands_for(np64(w), fmt, gw)
    ref = Q.product(xv, wv, None if b is None else np64(b), None if res is None else np64(res), act == dc.ACT_RELU6)
    extra = (0 if b is None else np.abs(np64(b))[None, :]) + (0 if res is None else np.abs(np64(res)))
    err = np.abs(np64(y.t) - ref)
    lim = bound(xv, wv, extra, ref, dtype, c_in)
    bad = err > lim
    assert not bad.any(), ("%d of %d" % (bad.sum(), bad.size), [(int(i), int(j), float(np64(y.t)[i, j]), float(ref[i, j])) for i, j in np.argwhere(bad)[:5]])
    rel = np.linalg.norm(np64(y.t) - ref) / max(np.linalg.norm(ref), 1e-30)
    assert rel <= (1e-5 if dtype == "f32" else 2.0 ** -8), rel
    return rel


PRODUCTS = [(128, 256, 256), (128, 64, 32), (1, 16, 8), (1, 1, 1), (5, 24, 144), (130, 320, 1280), (257, 1000, 1003), (16, 4096, 512), (1, 8192, 200), (384, 520, 300),
            (1000, 96, 64), (64, 33, 31), (129, 255, 257), (2048, 512, 2048), (3, 700, 40)]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("rows,c_in,c_out", PRODUCTS)
def test_product(rows, c_in, c_out, fmt, dtype):
    odd = (rows + c_in + c_out) % 2
    run_product(rows, c_in, c_out, fmt, dtype, bias=True, residual=bool(odd), act=dc.ACT_RELU6 if odd else dc.ACT_IDENTITY, forward=False)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("rows,c_in,c_out", [(1, 4096, 4096), (2, 24, 144), (7, 1003, 77), (16, 8192, 1024), (33, 640, 640), (64, 256, 1000), (600, 24, 144),
                                             (9, 20000, 64), (1, 40, 3), (300, 200, 72)])
def test_forward(rows, c_in, c_out, fmt, dtype):
    run_product(rows, c_in, c_out, fmt, dtype, bias=False, residual=True, act=dc.ACT_IDENTITY, forward=True)

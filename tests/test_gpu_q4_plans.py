"""4-bit products in every way that dc_q4_plan_query can answer: form, width of the tiles, clusters, accumulators, columns of tiles, weights that stay,
rows of y that begin on 16 bytes and that do not, one tile to a CTA or many, a ring that is filled once or many times -- in both formats.
test_q4_plans_host.py draws sizes and holds the lists here to what the estimate picks for them.

The reference is a product in 64 bits of the values that the quantised operands stand for, read back (exactly: see test_gpu_q4.py) and compared with the
oracle's in some rows.  An element may be off by what test_gpu_q4.py derives: 2^-23 K S of the sum, two roundings of fp32 behind it, and the result's own."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from oracle import q4_oracle as Q
from paper_2301_12187_b200 import dc
from tests.parity_util import Guarded

FMTS = [dc.MX4, dc.NV4]
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SMS = 148                                        # of the device that plans without a device are made for


def way(rows, c_in, c_out, fmt, dtype, forward):
    """The branches that a call of this size takes, as far as its plan tells."""
    p = dc.q4_plan(rows, c_in, c_out, fmt, dtype, forward)
    pairs = p.form == dc.Q4_PAIRS
    tiles_n = -(-c_out // p.tile_cols)
    tiles = -(-rows // (256 if pairs else 128)) * tiles_n
    turns = -(-tiles // (SMS // 2 if pairs else SMS // p.split))       # tiles of a CTA
    return ("%s%s" % (("tiles", "pairs", "few rows", "stream")[p.form], ", quantised apart" if forward and p.launches == 2 else ""),
            "mx4" if fmt == dc.MX4 else "nv4",
            "narrow" if p.tile_cols < 128 and tiles_n > 1 else "one scale tile" if p.tile_cols <= 128 else "two scale tiles",
            "cluster" if p.split > 1 else "alone", "%d accumulators" % p.accumulators,
            "columns" if p.columns else "rows and columns", "w stays" if p.w_stays else "w streamed",
            "rows of 16 bytes" if c_out * (4 if dtype == dc.F32 else 2) % 16 == 0 else "ragged rows",
            "one tile" if turns == 1 else "each accumulator once or twice" if turns <= 2 * p.accumulators else "many tiles",
            "ring once" if -(-c_in // 256) * turns <= p.stages * p.split else "ring again and again")


PRODUCTS = [
    # pairs of CTAs with several tiles each, of 256 and of 128 columns
    (6000, 2300, 4104), (25662, 2464, 1024), (1245, 1153, 2096), (1356, 2835, 1700), (1393, 3558, 5167), (604, 5236, 15060), (4372, 1423, 1600), (6961, 1291, 2024),
    (1095, 3317, 11169),
    # many tiles to a CTA, w kept and streamed, one scale tile and two
    (5200, 1100, 4100), (13056, 82, 2810), (51583, 88, 156), (16764, 335, 287), (9741, 1314, 168), (28749, 842, 138), (12675, 2394, 173), (31709, 1010, 176),
    (5000, 523, 3468), (1586, 23, 8566), (42571, 1070, 136), (1472, 1, 9780), (1044, 2615, 11680), (133, 24, 11616), (4032, 2100, 2704),
    # one column of tiles
    (9478, 1, 140), (19320, 2, 1), (32606, 13, 172), (130846, 1, 164), (72061, 21, 129), (114531, 1, 131), (122067, 15, 136), (84982, 381, 175),
    (32036, 3463, 153), (120292, 1010, 144), (177480, 728, 133), (104836, 2608, 179),
    # few rows
    (257, 1593, 69), (1, 465, 9868), (1, 3408, 12996), (3, 949, 9776),
]
FORWARDS = [(53, 4, 4), (1, 2088, 1), (1, 2068, 8), (1, 13573, 2), (126969, 8, 8), (43211, 4, 160), (23849, 4, 160), (110928, 8, 72), (73273, 20, 144), (103411, 16, 160),
            (200704, 24, 144), (1, 4096, 4096), (8, 1024, 520), (7, 68, 1277), (1, 11403, 1408), (36, 24, 208), (9, 20000, 64)]


def values_of(q):
    v = torch.empty(q.rows, q.cols, device="cuda")
    dc.q4_dequantize(q, v)
    return v.double()


def operands(rows, c_in, c_out, fmt, dtype, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed + rows * 7 + c_in * 3 + c_out)
    x = torch.randn(rows, c_in, generator=gen, device="cuda") * torch.exp(0.7 * torch.randn(c_in, generator=gen, device="cuda"))
    w = torch.randn(c_out, c_in, generator=gen, device="cuda") / c_in ** 0.5
    x = x.to(TYPES[dtype])
    out = []
    for t in (x, w):
        q = dc.Q4Matrix(*t.shape, fmt, 1.0 if fmt == dc.MX4 else dc.q4_tensor_scale(float(t.float().abs().max())))
        dc.q4_quantize(t, q)
        v = values_of(q)
        pick = sorted({0, t.shape[0] // 2, t.shape[0] - 1})
        assert (v[pick].cpu().numpy() == Q.stands_for(t[pick].double().cpu().numpy(), fmt, q.tensor_scale)).all()
        out += [q, v]
    bias = torch.randn(c_out, generator=gen, device="cuda")
    residual = torch.randn(rows, c_out, generator=gen, device="cuda").to(TYPES[dtype])
    return [x] + out + [bias, residual]


def check(y, xv, wv, bias, residual, act, dtype):
    ref, sums = xv @ wv.t(), xv.abs() @ wv.abs().t()
    for t in (bias, residual):
        if t is not None:
            ref += t.double()
            sums += t.double().abs()
    if act == dc.ACT_RELU6:
        ref.clamp_(0.0, 6.0)
    eps = torch.finfo(TYPES[dtype]).eps / 2
    limit = (sums + ref.abs()).mul_((xv.shape[1] + 3) * 2.0 ** -23).add_(ref.abs(), alpha=eps).add_(1e-37)
    err = (y.double() - ref).abs()
    bad = ~(err <= limit)
    assert not bad.any(), ("%d of %d" % (int(bad.sum()), bad.numel()), bad.nonzero()[:5].tolist(), y[bad][:5].tolist(), ref[bad][:5].tolist())


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("rows,c_in,c_out", PRODUCTS)
def test_product(rows, c_in, c_out, fmt, dtype):
    _, xq, xv, wq, wv, bias, residual = operands(rows, c_in, c_out, fmt, dtype, 1)
    ws = torch.zeros(dc.conv_workspace_bytes(), dtype=torch.uint8, device="cuda")
    for b, r, act in ((bias, None, dc.ACT_RELU6), (None, residual, dc.ACT_IDENTITY)):
        y = Guarded(torch, (rows, c_out), TYPES[dtype], fill=77.0)
        if r is not None and rows % 2 == 0:
            y.t.copy_(r)
        dc.q4_product(xq, wq, b, act, y.t if r is not None and rows % 2 == 0 else r, y.t, ws)
        assert dc.workspace_status(ws) == dc.OK
        y.check("result")
        check(y.t, xv, wv, b, r, act, dtype)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("rows,c_in,c_out", FORWARDS)
def test_forward(rows, c_in, c_out, fmt, dtype):
    x, xq, xv, wq, wv, bias, residual = operands(rows, c_in, c_out, fmt, dtype, 2)
    ws = torch.zeros(dc.q4_workspace_bytes(rows, c_in, fmt), dtype=torch.uint8, device="cuda")
    for b, r, act in ((None, None, dc.ACT_IDENTITY), (bias, None, dc.ACT_RELU6), (bias, residual, dc.ACT_IDENTITY)):
        y = Guarded(torch, (rows, c_out), TYPES[dtype], fill=77.0)
        dc.q4_forward(x, wq, xq.tensor_scale, b, act, r, y.t, ws)
        assert dc.workspace_status(ws) == dc.OK
        y.check("result")
        check(y.t, xv, wv, b, r, act, dtype)


@pytest.mark.parametrize("rows,c_in,c_out,dtype", [(6000, 2300, 4104, "bf16"), (25662, 2464, 1024, "f32"), (1393, 3558, 5167, "bf16"), (5200, 1100, 4100, "bf16")])
def test_many_tiles_give_the_same_bits_beside_other_streams(rows, c_in, c_out, dtype):
    """Pairs of CTAs that walk over several tiles, each with its two accumulators or its one, while two other streams run the same."""
    _, xq, _, wq, _, _, residual = operands(rows, c_in, c_out, dc.NV4, dtype, 3)
    streams = [torch.cuda.Stream() for _ in range(3)]
    ys = [[torch.empty(rows, c_out, dtype=TYPES[dtype], device="cuda") for _ in range(4)] for _ in streams]
    wss = [torch.zeros(dc.conv_workspace_bytes(), dtype=torch.uint8, device="cuda") for _ in streams]
    torch.cuda.synchronize()
    for i in range(4):
        for st, y, ws in zip(streams, ys, wss):
            dc.q4_product(xq, wq, None, dc.ACT_IDENTITY, residual, y[i], ws, stream=st)
    torch.cuda.synchronize()
    assert all(dc.workspace_status(ws) == dc.OK for ws in wss)
    for y in ys:
        for t in y:
            assert torch.equal(t, ys[0][0])

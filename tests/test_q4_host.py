"""4-bit matrices without a GPU: the layout, every refusal (before anything is launched), the binding's checks, and the oracle against the
definitions worked by hand."""
import ctypes as C

import numpy as np
import pytest

from oracle import q4_oracle as Q
from paper_2301_12187_b200 import dc

FAKE = 0x10000  # a 16-byte aligned, never dereferenced "device pointer"


def status_of(fn, *a):
    try:
        fn(*a)
    except dc.DcError as e:
        return e.status
    return dc.OK


@pytest.mark.parametrize("rows,cols,fmt,pitch,tiles,offset,nbytes", [
    (1, 1, dc.MX4, 32, 1, 256, 768),
    (1, 1, dc.NV4, 32, 1, 256, 768),
    (128, 24, dc.MX4, 32, 1, 4096, 4608),
    (129, 64, dc.NV4, 32, 1, 4352, 4352 + 2 * 512),
    (129, 65, dc.NV4, 64, 2, 8448, 8448 + 4 * 512),
    (4096, 4096, dc.NV4, 2048, 64, 4096 * 2048, 4096 * 2048 + 32 * 64 * 512),
    (300, 129, dc.MX4, 96, 2, 28928, 28928 + 3 * 2 * 512),
])
def test_layout(rows, cols, fmt, pitch, tiles, offset, nbytes):
    lay = dc.q4_layout(rows, cols, fmt)
    assert (lay.pitch, lay.tiles, lay.scale_offset, lay.bytes) == (pitch, tiles, offset, nbytes)
    assert dc.q4_workspace_bytes(rows, cols, fmt) == 256 + nbytes


def test_layout_of_large_matrices_passes_32_bits():
    lay = dc.q4_layout(1 << 30, 8192, dc.NV4)
    assert lay.scale_offset == (1 << 30) * 4096 and lay.bytes == lay.scale_offset + (1 << 23) * 128 * 512


def test_query_refuses():
    assert status_of(dc.q4_layout, 0, 8, dc.MX4) == dc.ERR_INVALID_ARG
    assert status_of(dc.q4_layout, -1, 8, dc.MX4) == dc.ERR_INVALID_ARG
    assert status_of(dc.q4_layout, 8, 0, dc.MX4) == dc.ERR_INVALID_ARG
    assert status_of(dc.q4_layout, 8, 8, 2) == dc.ERR_INVALID_ARG
    assert status_of(dc.q4_layout, (1 << 31) - 255, 8, dc.MX4) == dc.ERR_UNSUPPORTED
    assert status_of(dc.q4_layout, 8, (1 << 24) + 1, dc.MX4) == dc.ERR_UNSUPPORTED
    assert dc.lib().dc_q4_query(8, 8, 0, None) == dc.ERR_INVALID_ARG
    assert dc.lib().dc_q4_workspace_bytes(8, 8, 0, None) == dc.ERR_INVALID_ARG
    assert status_of(dc.q4_workspace_bytes, 0, 8, 0) == dc.ERR_INVALID_ARG


@pytest.mark.parametrize("name", ["dc_q4_quantize", "dc_q4_dequantize"])
def test_quantize_and_read_back_refuse(name):
    f = getattr(dc.lib(), name)

    def call(x=FAKE, rows=4, cols=8, stride=8, dtype=dc.BF16, fmt=dc.NV4, g=1.0, q=FAKE):
        if name == "dc_q4_quantize":
            return f(x, rows, cols, stride, dtype, fmt, g, q, None)
        return f(q, rows, cols, fmt, g, x, stride, dtype, None)

    bad = dc.ERR_INVALID_ARG
    assert call(x=None) == bad and call(q=None) == bad and call(rows=0) == bad and call(cols=0) == bad
    assert call(stride=7) == bad and call(dtype=2) == bad and call(fmt=-1) == bad
    for g in (0.0, -1.0, 3.0, 0.1, float("nan"), float("inf"), 2.0 ** -101, 2.0 ** 101, 1e-45):
        assert call(g=g) == bad, g
    assert call(fmt=dc.MX4, g=2.0) == bad
    assert call(x=FAKE + 8) == dc.ERR_ALIGNMENT and call(q=FAKE + 4) == dc.ERR_ALIGNMENT
    assert call(rows=1 << 31, stride=8) == dc.ERR_UNSUPPORTED


@pytest.mark.parametrize("forward", [False, True])
def test_products_refuse(forward):
    lib = dc.lib()
    size = dc.q4_workspace_bytes(4, 8, dc.NV4) if forward else dc.conv_workspace_bytes()

    def call(x=FAKE, rows=4, c_in=8, w=FAKE, c_out=16, fmt=dc.NV4, scale=1.0, bias=None, act=0, residual=None, y=FAKE, dtype=dc.BF16, ws=FAKE, n=size):
        if forward:
            return lib.dc_q4_forward(x, rows, c_in, w, c_out, fmt, scale, 1.0, bias, act, residual, y, dtype, ws, n, None)
        return lib.dc_q4_product(x, rows, c_in, w, c_out, fmt, scale, bias, act, residual, y, dtype, ws, n, None)

    bad = dc.ERR_INVALID_ARG
    assert call(x=None) == bad and call(w=None) == bad and call(y=None) == bad
    assert call(rows=0) == bad and call(c_in=0) == bad and call(c_out=0) == bad and call(fmt=5) == bad
    assert call(act=2) == bad and call(dtype=7) == bad
    assert call(scale=float("nan")) == bad and call(scale=float("inf")) == bad
    if forward:
        assert call(scale=3.0) == bad and call(fmt=dc.MX4, scale=2.0) == bad
    assert call(ws=None) == dc.ERR_WORKSPACE and call(n=255) == dc.ERR_WORKSPACE and call(n=size - 1) == dc.ERR_WORKSPACE
    for arg in ("x", "w", "y", "bias", "residual", "ws"):
        assert call(**{arg: FAKE + 4}) == dc.ERR_ALIGNMENT, arg


def test_binding_checks_shapes_and_types():
    torch = pytest.importorskip("torch")
    q = dc.Q4Matrix(6, 40, dc.NV4, 0.5, device="cpu")
    other = dc.Q4Matrix(6, 40, dc.MX4, device="cpu")
    w = dc.Q4Matrix(10, 40, dc.NV4, device="cpu")
    ws = torch.zeros(dc.q4_workspace_bytes(6, 40, dc.NV4), dtype=torch.uint8)
    for x in (torch.zeros(6, 41), torch.zeros(5, 40), torch.zeros(40, 6).t(), torch.zeros(3, 4, 40)[:, ::2][:, :, :40].transpose(0, 1)):
        with pytest.raises(ValueError):
            dc.q4_quantize(x, q, stream=_NullStream())
    with pytest.raises(ValueError):
        dc.q4_quantize(torch.zeros(6, 40, dtype=torch.float16), q, stream=_NullStream())
    y = torch.zeros(6, 10)
    with pytest.raises(ValueError):
        dc.q4_product(other, w, None, 0, None, y, ws, stream=_NullStream())
    for args in ((None, torch.zeros(6, 9)), (None, torch.zeros(6, 20)[:, ::2]), (torch.zeros(10, dtype=torch.bfloat16), y), (torch.zeros(9), y)):
        with pytest.raises(ValueError):
            dc.q4_product(q, w, args[0], 0, None, args[1], ws, stream=_NullStream())
    with pytest.raises(ValueError):
        dc.q4_product(q, w, None, 0, torch.zeros(6, 10, dtype=torch.bfloat16), y, ws, stream=_NullStream())
    with pytest.raises(ValueError):
        dc.q4_forward(torch.zeros(6, 40, dtype=torch.bfloat16), w, 1.0, None, 0, None, y, ws, stream=_NullStream())
    with pytest.raises(ValueError):
        dc.q4_forward(torch.zeros(6, 80)[:, ::2], w, 1.0, None, 0, None, y, ws, stream=_NullStream())


class _NullStream:
    cuda_stream = 0


def test_rows_at_one_distance():
    torch = pytest.importorskip("torch")
    rows = dc._rows_of
    assert rows(torch.zeros(2, 3, 4, 24), 24, "") == (24, 24)
    assert rows(torch.zeros(2, 3, 4, 40)[..., :24], 24, "") == (24, 40)
    assert rows(torch.zeros(24), 24, "") == (1, 24)
    assert rows(torch.zeros(1, 1, 1, 24), 24, "") == (1, 24)
    assert rows(torch.zeros(5, 1, 24), 24, "") == (5, 24)
    with pytest.raises(ValueError):
        rows(torch.zeros(4, 6, 24)[:, :3], 24, "")


def test_tensor_scale():
    assert dc.q4_tensor_scale(2688.0) == 1.0 and dc.q4_tensor_scale(2689.0) == 2.0 and dc.q4_tensor_scale(1344.0) == 0.5
    assert dc.q4_tensor_scale(0.0) == 1.0 and dc.q4_tensor_scale(float("nan")) == 1.0
    for top in (1e-3, 0.7, 5.0, 1e4):
        g = dc.q4_tensor_scale(top)
        assert np.log2(g) == np.round(np.log2(g)) and 224 < top / (6 * g) <= 448


def test_oracle_against_the_definition():
    # MX4: largest magnitude 5.0 -> 2^(2-2): codes are the values themselves, rounded
    x = np.zeros((1, 40))
    x[0, :8] = [5.0, -0.25, 0.26, 0.75, 1.25, 2.5, -3.5, 6e-3]
    x[0, 32] = 7.0                                                     # block of its own: 2^0, 7 is cut off at 6
    code, byte = Q.quantize(x, Q.MX4)
    assert byte.tolist() == [[127, 127]]
    assert code[0, :8].tolist() == [6, 8, 1, 2, 2, 4, 14, 0] and code[0, 32] == 7
    # NV4, g = 1/2: 9 / (6 / 2) = 3 = 1.5 * 2: byte 0x44; codes are value / 1.5
    x = np.zeros((1, 16))
    x[0, :3] = [9.0, 4.5, -1.5]
    code, byte = Q.quantize(x, Q.NV4, 0.5)
    assert byte[0, 0] == 0x44 and code[0, :3].tolist() == [7, 5, 10]
    assert Q.values(code, byte, Q.NV4, 0.5)[0, :3].tolist() == [9.0, 4.5, -1.5]
    # scale bytes are e4m3's own: 448 is 0x7e, the smallest one 2^-9
    assert Q.E4M3[0x7e] == 448.0 and Q.E4M3[1] == 2.0 ** -9 and len(Q.E4M3) == 127


def test_oracle_rounds_ties_to_even_codes():
    for fmt in (Q.MX4, Q.NV4):
        ties = np.array([[6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]])
        code, _ = Q.quantize(ties, fmt)
        assert code[0].tolist() == [7, 0, 2, 2, 4, 4, 6, 6]


def test_oracle_quantises_what_it_read_back_to_itself():
    r = np.random.default_rng(3)
    for fmt, g in ((Q.MX4, 1.0), (Q.NV4, 2.0 ** -8)):
        v = Q.stands_for(r.standard_normal((50, 96)), fmt, g)
        assert (Q.stands_for(v, fmt, g) == v).all()


def test_unpack_places_scales_as_the_header_says():
    rows, cols, fmt = 300, 200, dc.NV4
    lay = dc.q4_layout(rows, cols, fmt)
    buf = np.zeros(lay.bytes, dtype=np.uint8)
    r = np.random.default_rng(5)
    want = r.integers(0, 256, (rows, 13))
    for i in range(rows):
        for b in range(13):
            buf[lay.scale_offset + ((i // 128) * lay.tiles + b // 4) * 512 + (i % 32) * 16 + (i % 128) // 32 * 4 + b % 4] = want[i, b]
    buf[7 * lay.pitch + 3] = 0xA5
    code, byte = Q.unpack(buf, rows, cols, fmt)
    assert (byte[:rows, :13] == want).all() and code[7, 6] == 5 and code[7, 7] == 10


def test_plans():
    q = dc.q4_plan
    # few rows: in the product's launch, a cluster to a tile where tiles alone would leave SMs idle; many rows: apart, except of narrow layers
    p = q(1, 4096, 4096, dc.NV4, dc.BF16, True)
    assert p.form == dc.Q4_FEW_ROWS and p.launches == 1 and p.split > 1
    assert q(64, 4096, 4096, dc.NV4, dc.BF16, True).launches == 2
    assert q(16, 8192, 8192, dc.MX4, dc.BF16, True).launches == 2
    p = q(200704, 24, 144, dc.MX4, dc.BF16, True)
    assert p.form == dc.Q4_STREAM and p.launches == 1 and p.tile_cols == 144 and p.w_stays
    p = q(8192, 8192, 8192, dc.NV4, dc.BF16, False)
    assert p.form == dc.Q4_PAIRS and p.tile_cols == 256 and p.stages >= 5
    p = q(6272, 320, 1280, dc.MX4, dc.BF16, False)
    assert p.form == dc.Q4_TILES and p.accumulators == 3 and p.columns and p.w_stays
    assert status_of(q, 0, 8, 8, dc.MX4, dc.BF16, False) == dc.ERR_INVALID_ARG
    assert status_of(q, 8, 8, 8, dc.MX4, 5, False) == dc.ERR_INVALID_ARG
    assert dc.lib().dc_q4_plan_query(8, 8, 8, 0, 1, 0, None) == dc.ERR_INVALID_ARG


def test_every_size_has_a_plan():
    r = np.random.default_rng(1)
    for _ in range(4000):
        rows, c_in, c_out = (int(np.exp(r.uniform(0, np.log(n)))) for n in (1 << 24, 1 << 17, 1 << 17))
        for fmt in (dc.MX4, dc.NV4):
            for dtype in (dc.F32, dc.BF16):
                for forward in (False, True):
                    p = dc.q4_plan(rows, c_in, c_out, fmt, dtype, forward)
                    assert p.stages >= 2 and 1 <= p.split <= 8 and p.tile_cols in range(16, 257, 16), (rows, c_in, c_out, fmt, dtype)
                    assert p.accumulators * p.tile_cols <= 512 - 32


def test_the_gpu_tests_reach_every_form():
    torch = pytest.importorskip("torch")
    from tests import test_gpu_q4 as t
    seen = {}
    for rows, c_in, c_out in t.FORMS + t.PRODUCTS:
        for fmt in (dc.MX4, dc.NV4):
            for dtype in (dc.F32, dc.BF16):
                p = dc.q4_plan(rows, c_in, c_out, fmt, dtype, False)
                whole = c_out * (4 if dtype == dc.F32 else 2) % 16 == 0
                for what in ("pairs %d" % p.tile_cols if p.form == dc.Q4_PAIRS else "split" if p.split > 1 else "tiles %d" % p.accumulators,
                             "columns, w %s" % ("stays" if p.w_stays else "not") if p.columns else "", "two scale tiles" if p.tile_cols > 128 else ""):
                    seen.setdefault((what, whole), (rows, c_in, c_out))
    for what in ("pairs 256", "split", "tiles 1", "tiles 3", "columns, w stays", "two scale tiles"):
        for whole in (False, True):
            assert (what, whole) in seen, (what, whole)
    forms = {dc.q4_plan(r, i, o, f, d, True).form for r, i, o in t.FORWARD_FORMS for f in (0, 1) for d in (0, 1)}
    assert {dc.Q4_FEW_ROWS, dc.Q4_STREAM, dc.Q4_TILES} <= forms


@pytest.mark.parametrize("native", [True, False])
def test_binding_refuses_a_buffer_that_does_not_hold_its_matrix(native, monkeypatch):
    """A matrix's buffer may be replaced by the caller, by a loaded one for instance."""
    torch = pytest.importorskip("torch")
    dc.lib()
    if not native:
        monkeypatch.setattr(dc, "_native", dc._NoNative)
    x, y, ws = torch.zeros(4, 40), torch.zeros(4, 16), torch.zeros(1 << 16, dtype=torch.uint8)
    good_x, good_w = dc.Q4Matrix(4, 40, dc.NV4, device="cpu"), dc.Q4Matrix(16, 40, dc.NV4, device="cpu")
    n = int(good_w.layout.bytes)
    for data in (torch.zeros(n - 1, dtype=torch.uint8), torch.zeros(2 * n, dtype=torch.uint8)[::2]):
        w = dc.Q4Matrix(16, 40, dc.NV4, device="cpu")
        w.data = data
        for call in (lambda: dc.q4_quantize(torch.zeros(16, 40), w), lambda: dc.q4_dequantize(w, torch.zeros(16, 40)),
                     lambda: dc.q4_product(good_x, w, None, 0, None, y, ws), lambda: dc.q4_product(w, good_x, None, 0, None, torch.zeros(16, 4), ws),
                     lambda: dc.q4_forward(x, w, 1.0, None, 0, None, y, ws)):
            with pytest.raises(ValueError, match="buffer"):
                call()


def test_narrow_tiles_are_for_few_tiles_of_fp32_or_ragged_rows():
    torch = pytest.importorskip("torch")
    from tests import test_gpu_q4 as t
    seen = set()
    for rows, c_in, c_out in t.NARROW:
        for fmt in (dc.MX4, dc.NV4):
            for dtype in (dc.F32, dc.BF16):
                p = dc.q4_plan(rows, c_in, c_out, fmt, dtype, False)
                if p.tile_cols < 128:
                    assert p.form == dc.Q4_TILES and p.split == 1 and p.accumulators == 1 and not p.columns
                    seen.add((p.tile_cols, fmt, dtype))
    assert seen >= {(n, f, d) for n, d in ((32, dc.F32), (32, dc.BF16), (64, dc.F32)) for f in (0, 1)}
    # many tiles, and bf16 rows that begin on 16 bytes: whole scale tiles
    for rows, c_in, c_out in ((128, 4096, 4096), (256, 1280, 1000), (6272, 320, 1280), (20000, 200, 520)):
        assert dc.q4_plan(rows, c_in, c_out, dc.NV4, dc.BF16, False).tile_cols >= 128
    assert dc.q4_plan(20000, 200, 521, dc.NV4, dc.F32, False).tile_cols >= 128


@pytest.mark.parametrize("fmt", [dc.NV4])
def test_forward_refuses_tensor_scales_whose_product_fp32_does_not_hold(fmt):
    """Sums of codes times block scales pass 2^22: a product of scales that fp32 rounds to 0 would leave bias + residual of results that it can hold."""
    size = dc.q4_workspace_bytes(4, 64, fmt)

    def call(x_scale, w_scale):
        return dc.lib().dc_q4_forward(FAKE, 4, 64, FAKE, 16, fmt, x_scale, w_scale, None, 0, None, FAKE, dc.BF16, FAKE, size, None)

    for a, b in ((100, 28), (100, 100), (-100, -50), (-50, -100), (-100, -60), (-100, -100)):
        assert call(2.0 ** a, 2.0 ** b) == dc.ERR_INVALID_ARG, (a, b)


@pytest.mark.parametrize("native", [True, False])
def test_product_refuses_tensor_scales_whose_product_fp32_does_not_hold(native, monkeypatch):
    torch = pytest.importorskip("torch")
    dc.lib()
    if not native:
        monkeypatch.setattr(dc, "_native", dc._NoNative)
    y, ws = torch.zeros(4, 16), torch.zeros(1 << 16, dtype=torch.uint8)
    # the last one: subnormal in fp32, with bits that it does not have there
    for a, b in ((2.0 ** -100, 2.0 ** -50), (2.0 ** -100, -(2.0 ** -60)), (2.0 ** -100, 2.0 ** -100), (2.0 ** -60, 1e-300), (1.25 * 2.0 ** -100, 2.0 ** -48)):
        x, w = dc.Q4Matrix(4, 40, dc.NV4, a, device="cpu"), dc.Q4Matrix(16, 40, dc.NV4, b, device="cpu")
        with pytest.raises(ValueError, match="tensor scales"):
            dc.q4_product(x, w, None, 0, None, y, ws, stream=_NullStream())


def all_bf16_magnitudes():
    return (np.arange(0x7f80, dtype=np.uint32) << 16).view(np.float32)


@pytest.mark.parametrize("g", [1.0, 2.0 ** -8, 2.0 ** 13, 2.0 ** -100, 2.0 ** 100])
def test_oracle_scales_against_the_quotient_of_real_arithmetic(g):
    """NV4's scale is a product in fp32 with 1 / (6 g): of a block of bf16 values the same byte as the quotient's, of fp32 values unless that lies within
    2^-23 of a border.  (1 / (6 g) is rounded by 2^-25 of it, g being a power of two, and the product by at most 2^-24; a product below 2^-126, which loses
    more, is far below the first border, 2^-10.)"""
    top = all_bf16_magnitudes().astype(np.float64)
    x = np.zeros((top.size, 16))
    x[:, 3] = -top
    assert (Q.quantize(x, Q.NV4, g)[1][:, 0] == Q.exact_scale_byte(top, g)).all()
    r = np.random.default_rng(9)
    mid = (Q.E4M3[1:] + Q.E4M3[:-1]) / 2
    near = np.repeat((6.0 * g * mid).astype(np.float32)[:, None], 9, 1)                # borders, and the next numbers on either side
    for i in range(4):
        near[:, i] = np.nextafter(near[:, i + 1] if i else near[:, 8], np.float32(0))
        near[:, 4 + i] = np.nextafter(near[:, 3 + i] if i else near[:, 8], np.float32(np.inf))
    top = np.concatenate([near.ravel(), (np.exp(r.uniform(-8, 7, 20000)) * 6 * g).astype(np.float32)]).astype(np.float64)
    x = np.zeros((top.size, 16))
    x[:, 15] = top
    byte, exact = Q.quantize(x, Q.NV4, g)[1][:, 0], Q.exact_scale_byte(top, g)
    off = byte != exact
    border = mid[np.minimum(byte, exact)[off]]
    assert (np.abs(byte - exact) <= 1).all() and (np.abs(top[off] / (6 * g) / border - 1) <= 2.0 ** -23).all()

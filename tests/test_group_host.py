"""Grouped products and adapters without a GPU: every refusal (before anything is launched), sizes of buffers, and the binding's checks."""
import ctypes as C

import pytest

torch = pytest.importorskip("torch")

from paper_2301_12187_b200 import dc

FAKE = 0x10000  # a 16-byte aligned, never dereferenced "device pointer"
BIG = 1 << 40


def adapters(count=3, rank=8, a=FAKE, b=FAKE, scale=None):
    return dc.AdapterSet(count, rank, a, b, scale)


def forward(x=FAKE, rows=4, c_in=8, off=FAKE, groups=2, w=FAKE, c_out=8, bias=None, act=0, y=FAKE, dtype=dc.BF16, ws=FAKE, size=BIG):
    return dc.lib().dc_group_forward(x, rows, c_in, off, groups, w, c_out, bias, act, y, dtype, ws, size, None)


def backward(dy=FAKE, x=FAKE, rows=4, c_in=8, off=FAKE, groups=2, w=FAKE, c_out=8, dx=FAKE, dw=FAKE, db=FAKE, dtype=dc.BF16, ws=FAKE, size=BIG):
    return dc.lib().dc_group_backward(dy, x, rows, c_in, off, groups, w, c_out, dx, dw, db, dtype, ws, size, None)


def adapter_forward(x=FAKE, rows=4, c_in=8, w=FAKE, c_out=8, ad="ok", off=FAKE, which=FAKE, runs=2, bias=None, act=0, residual=None, saved=FAKE,
                    y=FAKE, dtype=dc.BF16, ws=FAKE, size=BIG):
    ad = adapters() if ad == "ok" else ad
    return dc.lib().dc_adapter_forward(x, rows, c_in, w, c_out, C.byref(ad) if ad is not None else None, off, which, runs, bias, act, residual,
                                       saved, y, dtype, ws, size, None)


def adapter_backward(dy=FAKE, x=FAKE, rows=4, c_in=8, w=FAKE, c_out=8, ad="ok", off=FAKE, which=FAKE, runs=2, saved=FAKE, dx=FAKE, da=FAKE,
                     db=FAKE, dtype=dc.BF16, ws=FAKE, size=BIG):
    ad = adapters() if ad == "ok" else ad
    return dc.lib().dc_adapter_backward(dy, x, rows, c_in, w, c_out, C.byref(ad) if ad is not None else None, off, which, runs, saved, dx, da, db,
                                        dtype, ws, size, None)


EVERY = [forward, backward, adapter_forward, adapter_backward]


@pytest.mark.parametrize("call", EVERY)
def test_sizes_and_types_are_refused(call):
    bad, no = dc.ERR_INVALID_ARG, dc.ERR_UNSUPPORTED
    assert call(rows=-1) == bad and call(c_in=0) == bad and call(c_out=0) == bad and call(c_in=-8) == bad
    assert call(dtype=2) == bad and call(dtype=-1) == bad
    assert call(rows=(1 << 30) + 1) == no and call(c_in=(1 << 20) + 1) == no and call(c_out=(1 << 20) + 1) == no
    assert call(off=None) == bad
    assert call(ws=None) == dc.ERR_WORKSPACE and call(size=255) == dc.ERR_WORKSPACE and call(size=0) == dc.ERR_WORKSPACE
    assert call(ws=FAKE + 8) == dc.ERR_ALIGNMENT and call(off=FAKE + 2) == dc.ERR_ALIGNMENT and call(w=FAKE + 4) == dc.ERR_ALIGNMENT


def test_group_refuses():
    bad, no, off16 = dc.ERR_INVALID_ARG, dc.ERR_UNSUPPORTED, dc.ERR_ALIGNMENT
    for call in (forward, backward):
        assert call(groups=0) == bad and call(groups=(1 << 20) + 1) == no
    assert forward(act=2) == bad and forward(act=-1) == bad
    assert forward(x=None) == bad and forward(y=None) == bad and forward(w=None) == bad
    assert forward(x=FAKE + 2) == off16 and forward(y=FAKE + 8) == off16 and forward(bias=FAKE + 4) == off16
    assert backward(dy=None) == bad and backward(w=None) == bad and backward(x=None) == bad
    assert backward(dx=None, dw=None, db=None) == bad
    for name in ("dy", "x", "dx", "dw", "db"):
        assert backward(**{name: FAKE + 4}) == off16


def test_adapter_refuses():
    bad, no, off16 = dc.ERR_INVALID_ARG, dc.ERR_UNSUPPORTED, dc.ERR_ALIGNMENT
    for call in (adapter_forward, adapter_backward):
        assert call(ad=None) == bad
        assert call(ad=adapters(count=0)) == bad and call(ad=adapters(rank=0)) == bad
        assert call(ad=adapters(rank=129)) == no and call(ad=adapters(count=(1 << 20) + 1)) == no
        assert call(ad=adapters(a=None)) == bad and call(ad=adapters(b=None)) == bad
        assert call(ad=adapters(a=FAKE + 8)) == off16 and call(ad=adapters(scale=FAKE + 1)) == off16
        assert call(runs=-1) == bad and call(runs=(1 << 20) + 1) == no and call(which=None) == bad and call(which=FAKE + 2) == off16
    assert adapter_forward(act=7) == bad and adapter_forward(x=None) == bad and adapter_forward(y=None) == bad and adapter_forward(saved=None) == bad
    for name in ("x", "y", "saved", "residual", "bias"):
        assert adapter_forward(**{name: FAKE + 4}) == off16
    assert adapter_backward(dy=None) == bad and adapter_backward(dx=None, da=None, db=None) == bad
    assert adapter_backward(x=None) == bad and adapter_backward(saved=None) == bad
    for name in ("dy", "x", "saved", "dx", "da", "db"):
        assert adapter_backward(**{name: FAKE + 4}) == off16
    # a workspace without room for u
    n = C.c_size_t(0)
    assert dc.lib().dc_adapter_workspace_bytes(1000, 8, 8, C.byref(adapters()), dc.BF16, C.byref(n)) == dc.OK and n.value >= 256 + 1000 * 16 * 4
    assert adapter_backward(rows=1000, size=n.value - 1) == dc.ERR_WORKSPACE


def test_calls_without_rows_launch_nothing():
    """No GPU here: a launch would fail."""
    assert forward(rows=0, x=None, y=None) == dc.OK
    assert adapter_forward(rows=0, x=None, y=None, saved=None) == dc.OK
    assert adapter_forward(rows=0, x=None, y=None, saved=None, runs=0, which=None) == dc.OK
    assert backward(rows=0, dy=None, x=None, dx=None, dw=None, db=None) == dc.OK
    assert adapter_backward(rows=0, dy=None, x=None, dx=None, da=None, db=None, saved=None) == dc.OK


def test_buffer_sizes():
    n = C.c_size_t(0)
    for rank, pad in ((1, 16), (16, 16), (17, 32), (128, 128)):
        for dtype, each in ((dc.F32, 6), (dc.BF16, 4)):
            assert dc.adapter_saved_bytes(1000, rank, dtype) == 1000 * pad * each
    assert dc.lib().dc_adapter_saved_bytes(1 << 30, 128, dc.BF16, C.byref(n)) == dc.OK and n.value == 1 << 39
    assert dc.lib().dc_adapter_saved_bytes(-1, 8, dc.BF16, C.byref(n)) == dc.ERR_INVALID_ARG
    assert dc.lib().dc_adapter_saved_bytes(8, 129, dc.BF16, C.byref(n)) == dc.ERR_UNSUPPORTED
    assert dc.lib().dc_adapter_saved_bytes(8, 8, 3, C.byref(n)) == dc.ERR_INVALID_ARG
    assert dc.lib().dc_adapter_saved_bytes(8, 8, dc.F32, None) == dc.ERR_INVALID_ARG
    assert dc.lib().dc_group_workspace_bytes(8, 2, 8, 8, dc.F32, None) == dc.ERR_INVALID_ARG
    assert dc.group_workspace_bytes(0, 1, 1, 1, dc.BF16) >= 256


@pytest.fixture
def cpu(monkeypatch):
    """Tensors of no GPU pass for those of the current device, so that the binding's other checks are reached."""
    monkeypatch.setattr(dc, "_here", lambda *a: None)

    class Lib:
        def __getattr__(self, name):
            raise AssertionError("%s was called" % name)

    real = dc.lib()
    monkeypatch.setattr(dc, "_lib", Lib())
    Lib.dc_adapter_saved_bytes = staticmethod(real.dc_adapter_saved_bytes)      # sizes are asked for


def test_binding_refuses_what_does_not_fit(cpu):
    z = torch.zeros
    off, ws = z(3, dtype=torch.int32), z(256, dtype=torch.uint8)
    good = dict(x=z(4, 8), offsets=off, w=z(2, 6, 8), bias=z(2, 6), act=0, y=z(4, 6), workspace=ws)
    for change in (dict(x=z(4, 8, dtype=torch.bfloat16)), dict(y=z(4, 7)), dict(y=z(3, 6)), dict(w=z(6, 8)), dict(w=z(2, 8, 6).transpose(1, 2)),
                   dict(bias=z(6)), dict(bias=z(2, 6, dtype=torch.bfloat16)), dict(offsets=z(3, dtype=torch.int64)), dict(offsets=z(2, dtype=torch.int32)),
                   dict(x=z(4, 16)[:, ::2])):
        with pytest.raises(ValueError):
            dc.group_forward(**{**good, **change})
    back = dict(dy=z(4, 6), x=z(4, 8), offsets=off, w=z(2, 6, 8), dx=z(4, 8), dw=z(2, 6, 8), db=z(2, 6), workspace=ws)
    for change in (dict(dx=z(4, 6)), dict(dw=z(2, 8, 6)), dict(db=z(6)), dict(x=z(5, 8)), dict(dw=z(2, 6, 8, dtype=torch.bfloat16)),
                   dict(db=z(2, 6, dtype=torch.bfloat16)), dict(dy=z(4, 12)[:, :6])):
        with pytest.raises(ValueError):
            dc.group_backward(**{**back, **change})
    with pytest.raises(ValueError):
        dc.Adapters(z(2, 4, 8), z(2, 6, 5))
    with pytest.raises(ValueError):
        dc.Adapters(z(2, 4, 8), z(3, 6, 4))
    with pytest.raises(ValueError):
        dc.Adapters(z(2, 4, 8), z(2, 6, 4), z(3))
    with pytest.raises(ValueError):
        dc.Adapters(z(2, 4, 8), z(2, 4, 6).transpose(1, 2))
    ad = dc.Adapters(z(2, 4, 8), z(2, 6, 4), z(2))
    which, saved = z(2, dtype=torch.int32), z(4 * 96, dtype=torch.uint8)
    good = dict(x=z(4, 8), w=z(6, 8), adapters=ad, offsets=off, which=which, bias=z(6), act=0, residual=z(4, 6), saved=saved, y=z(4, 6), workspace=ws)
    for change in (dict(w=z(8, 6)), dict(x=z(4, 8, dtype=torch.bfloat16)), dict(offsets=z(4, dtype=torch.int32)), dict(which=z(2, dtype=torch.int64)),
                   dict(saved=saved[:-1]), dict(bias=z(8)), dict(residual=z(4, 8)), dict(y=z(5, 6))):
        with pytest.raises(ValueError):
            dc.adapter_forward(**{**good, **change})
    back = dict(dy=z(4, 6), x=z(4, 8), w=z(6, 8), adapters=ad, offsets=off, which=which, saved=saved, dx=z(4, 8), da=z(2, 4, 8), db=z(2, 6, 4), workspace=ws)
    for change in (dict(da=z(2, 8, 4)), dict(db=z(2, 4, 6)), dict(dx=z(4, 6)), dict(x=z(3, 8)), dict(da=z(2, 4, 8, dtype=torch.bfloat16)), dict(saved=saved[:100])):
        with pytest.raises(ValueError):
            dc.adapter_backward(**{**back, **change})

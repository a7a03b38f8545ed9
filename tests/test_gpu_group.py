"""Grouped products and adapters on the GPU against the formulas in 64 bits, element by element.

Tolerance of an element.  Products of two bf16 or fp32 numbers enter sums in fp32: each of the K additions of a sum loses at most 2^-23 of
the sum S of its terms' magnitudes (additions that cut off) and each product of fp32 numbers 2^-24 of itself, so a sum may be off by (K + 1) 2^-23 S.
Behind it come up to three roundings of fp32 (scale, bias, residual: 2^-23 of the magnitudes added, together with K + 4 in the place of K + 1) and the
rounding to the result's type, finfo.eps / 2 of the value.  What a row keeps of an adapter (t, u) is a sum as above, of magnitudes T, held in
fp32 or in two bf16 terms, which leaves 2^-16 of it at most (each of the two roundings halves of a last place: 2^-9 of 2^-9, with margin 2^-16); of
what is made of it, each term may then be off by that share of its own magnitude.
A gradient is also held against differences of the 64-bit forward formula."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2301_12187_b200 import dc
from tests.group_sizes import ADAPTER_FORMS, GROUP_FORMS, spread
from tests.parity_util import Guarded

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
U = 2.0 ** -23


def rand(*shape, seed, dtype, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def check(got, want, slack, what):
    """`slack`: what sums may lose; the result's rounding is added."""
    got = got.double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    room = slack + half_step_of(got, want)
    bad = ~((got - want).abs() <= room)
    assert not bool(bad.any()), "%s: %d of %d off, first at %s: %r, not %r (room %.3g)" % (
        what, int(bad.sum()), bad.numel(), bad.nonzero()[0].tolist(), float(got[bad][0]), float(want[bad][0]), float(room[bad][0]))


_TYPE = {}


def half_step_of(got, want):
    return want.abs() * _TYPE["eps"] * 1.0001 + 1e-37


def of_type(dtype):
    _TYPE["eps"] = half_step(dtype)


def runs_of(offsets):
    o = offsets.tolist()
    return list(zip(o[:-1], o[1:]))


def group_want(x, off, w, bias, act):
    """(y, slack, mask of rows that belong to a group), 64 bits."""
    x, rows = x.double(), x.shape[0]
    y = torch.zeros(rows, w.shape[1], dtype=torch.float64, device="cuda")
    s, mine = torch.zeros_like(y), torch.zeros(rows, dtype=torch.bool, device="cuda")
    k = x.shape[1]
    for g, (lo, hi) in enumerate(runs_of(off)):
        wg = w[g].double()
        y[lo:hi] = x[lo:hi] @ wg.t()
        s[lo:hi] = x[lo:hi].abs() @ wg.abs().t()
        if bias is not None:
            y[lo:hi] += bias[g].double()
            s[lo:hi] += bias[g].double().abs()
        mine[lo:hi] = True
    return (y.clamp(0, 6) if act else y), (k + 4) * U * s, mine


def offsets_of(sizes):
    return torch.tensor(np.concatenate([[0], np.cumsum(sizes)]).tolist(), dtype=torch.int32, device="cuda")


def workspace(nbytes):
    g = Guarded(torch, (nbytes,), torch.uint8, fill=0)
    return g


# sizes of groups; rows behind the last one; c_in, c_out
GROUPS = [
    ([1], 0, 8, 8),
    ([1], 0, 1, 1),
    ([3, 0, 5], 2, 64, 64),
    ([0, 0, 0, 7], 3, 72, 40),
    ([1, 1, 1, 1, 1, 1, 1, 1], 0, 128, 136),
    ([17, 1, 64, 65], 5, 200, 264),
    ([130, 127, 0, 129, 1], 1, 96, 512),
    ([300], 0, 1000, 320),
    ([5, 9, 33], 4, 65, 131),
    ([200, 3], 0, 67, 300),
    ([2] * 40 + [0] * 30 + [9], 7, 256, 192),
    ([16, 16, 31, 15], 0, 1024, 128),
    ([700, 260, 515], 9, 520, 776),
    ([2500, 1, 0, 1303], 5, 1032, 2056),         # pairs of CTAs
    ([1900, 1501], 3, 1031, 1100),
] + [(spread(rows, n, i), 0, c_in, c_out) for i, (rows, n, c_in, c_out) in enumerate(GROUP_FORMS)]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("case", range(len(GROUPS)))
def test_group_forward(case, dtype):
    sizes, tail, c_in, c_out = GROUPS[case]
    dt, rows, n = TYPES[dtype], sum(sizes) + tail, len(sizes)
    of_type(dt)
    for bias_too, act in ((False, 0), (True, 1)):
        x, w = rand(rows, c_in, seed=case, dtype=dt), rand(n, c_out, c_in, seed=case + 50, dtype=dt, scale=2.0 / c_in ** 0.5)
        bias = rand(n, c_out, seed=case + 99, dtype=torch.float32) if bias_too else None
        off = offsets_of(sizes)
        want, slack, mine = group_want(x, off, w, bias, act)
        y, ws = Guarded(torch, (rows, c_out), dt, fill=77.0), workspace(dc.group_workspace_bytes(rows, n, c_in, c_out, dc.dtype_code(dt)))
        if tail:
            x[-tail:] = float("nan")             # rows of no group
        dc.group_forward(x, off, w, bias, act, y.t, ws.t)
        torch.cuda.synchronize()
        y.check("y"), ws.check("workspace")
        assert dc.workspace_status(ws.t) == dc.OK
        check(y.t[mine], want[mine], slack[mine], "y")
        assert bool((y.t[~mine] == 77.0).all())


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("case", range(len(GROUPS)))
def test_group_backward(case, dtype):
    sizes, tail, c_in, c_out = GROUPS[case]
    dt, rows, n = TYPES[dtype], sum(sizes) + tail, len(sizes)
    of_type(dt)
    x, dy = rand(rows, c_in, seed=case + 3, dtype=dt), rand(rows, c_out, seed=case + 4, dtype=dt)
    w = rand(n, c_out, c_in, seed=case + 5, dtype=dt, scale=2.0 / c_in ** 0.5)
    if tail:
        x[-tail:] = float("nan")
        dy[-tail:] = float("inf")
    off = offsets_of(sizes)
    dx, dw = Guarded(torch, (rows, c_in), dt, fill=55.0), Guarded(torch, (n, c_out, c_in), dt, fill=float("nan"))
    db, ws = Guarded(torch, (n, c_out), torch.float32, fill=float("nan")), workspace(dc.group_workspace_bytes(rows, n, c_in, c_out, dc.dtype_code(dt)))
    dc.group_backward(dy, x, off, w, dx.t, dw.t, db.t, ws.t)
    torch.cuda.synchronize()
    for g in (dx, dw, db, ws):
        g.check("group_backward")
    assert dc.workspace_status(ws.t) == dc.OK
    mine = torch.zeros(rows, dtype=torch.bool, device="cuda")
    for g, (lo, hi) in enumerate(runs_of(off)):
        a, b, wg = dy[lo:hi].double(), x[lo:hi].double(), w[g].double()
        check(dx.t[lo:hi], a @ wg, (c_out + 4) * U * (a.abs() @ wg.abs()), "dx")
        check(dw.t[g], a.t() @ b, (hi - lo + 4) * U * (a.abs().t() @ b.abs()), "dw")
        assert bool(((db.t[g].double() - a.sum(0)).abs() <= (hi - lo + 4) * U * a.abs().sum(0)).all())
        mine[lo:hi] = True
    assert bool((dx.t[~mine] == 55.0).all())


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("most", [1, 9, 40])
def test_more_runs_than_one_look_finds(most, dtype):
    """1500 groups of up to `most` rows, many of them empty: tiles are found by walking over the runs, and a CTA has several."""
    dt, n, c_in, c_out = TYPES[dtype], 1500, 24, 72
    of_type(dt)
    g = torch.Generator().manual_seed(most)
    sizes = torch.randint(0, most + 1, (n,), generator=g).tolist()
    rows, off = sum(sizes), offsets_of(sizes)
    of = torch.repeat_interleave(torch.arange(n), torch.tensor(sizes)).cuda()
    x, dy, w = rand(rows, c_in, seed=1, dtype=dt), rand(rows, c_out, seed=2, dtype=dt), rand(n, c_out, c_in, seed=3, dtype=dt)
    ws = workspace(dc.group_workspace_bytes(rows, n, c_in, c_out, dc.dtype_code(dt)))
    y, dx, dw = Guarded(torch, (rows, c_out), dt, fill=7.0), Guarded(torch, (rows, c_in), dt, fill=7.0), Guarded(torch, (n, c_out, c_in), dt, fill=7.0)
    db = Guarded(torch, (n, c_out), torch.float32, fill=7.0)
    dc.group_forward(x, off, w, None, 0, y.t, ws.t)
    dc.group_backward(dy, x, off, w, dx.t, dw.t, db.t, ws.t)
    ad, which = dc.Adapters(w[:40, :8].contiguous(), w[:40, :, :8].contiguous()), torch.arange(n, dtype=torch.int32, device="cuda") % 41 - 1
    saved, z, aws = ad.saved(rows), Guarded(torch, (rows, c_out), dt, fill=7.0), workspace(dc.adapter_workspace_bytes(rows, c_in, c_out, ad, ad.dtype))
    dc.adapter_forward(x, w[0].contiguous(), ad, off, which, None, 0, None, saved, z.t, aws.t)
    torch.cuda.synchronize()
    for q in (y, dx, dw, db, z, ws, aws):
        q.check("many runs")
    assert dc.workspace_status(ws.t) == dc.OK and dc.workspace_status(aws.t) == dc.OK
    xd, dd, wr = x.double(), dy.double(), w.double()[of]
    check(y.t, torch.einsum("rk,rok->ro", xd, wr), (c_in + 4) * U * torch.einsum("rk,rok->ro", xd.abs(), wr.abs()), "y")
    check(dx.t, torch.einsum("ro,rok->rk", dd, wr), (c_out + 4) * U * torch.einsum("ro,rok->rk", dd.abs(), wr.abs()), "dx")
    each = torch.einsum("ro,rk->rok", dd, xd)
    sums, room = torch.zeros(n, c_out, c_in, dtype=torch.float64, device="cuda"), torch.zeros(n, c_out, c_in, dtype=torch.float64, device="cuda")
    check(dw.t, sums.index_add_(0, of, each), (most + 4) * U * room.index_add_(0, of, each.abs()), "dw")
    sums, room = torch.zeros(n, c_out, dtype=torch.float64, device="cuda"), torch.zeros(n, c_out, dtype=torch.float64, device="cuda")
    assert bool(((db.t.double() - sums.index_add_(0, of, dd)).abs() <= (most + 4) * U * room.index_add_(0, of, dd.abs())).all())
    want, slack = torch.zeros(rows, c_out, dtype=torch.float64, device="cuda"), (c_in + 16) * U * (xd.abs() @ w[0].double().abs().t())
    a, b, mine = ad.a.double(), ad.b.double(), which.long()[of]
    for i in range(40):
        r = mine == i
        t, m = xd[r] @ a[i].t(), xd[r].abs() @ a[i].abs().t()
        want[r] = t @ b[i].t()
        slack[r] += ((c_in + 4) * U * m + keeps(dt) * t.abs()) @ b[i].abs().t() + (c_in + 24) * U * (t.abs() @ b[i].abs().t())
    check(z.t, want + xd @ w[0].double().t(), slack, "z")


def test_group_backward_parts_alone():
    """Each gradient without the others, and without what it does not need, gives the same bits."""
    sizes, c_in, c_out = [33, 0, 130], 72, 264
    x, dy = rand(163, c_in, seed=1, dtype=torch.bfloat16), rand(163, c_out, seed=2, dtype=torch.bfloat16)
    w, off = rand(3, c_out, c_in, seed=3, dtype=torch.bfloat16), offsets_of(sizes)
    ws = torch.zeros(dc.group_workspace_bytes(163, 3, c_in, c_out, dc.BF16), dtype=torch.uint8, device="cuda")
    dx, dw, db = torch.zeros_like(x), torch.zeros_like(w), torch.zeros(3, c_out, device="cuda")
    dc.group_backward(dy, x, off, w, dx, dw, db, ws)
    dx1, dw1, db1 = torch.ones_like(x), torch.ones_like(w), torch.ones(3, c_out, device="cuda")
    dc.group_backward(dy, None, off, w, dx1, None, None, ws)
    dc.group_backward(dy, x, off, w, None, dw1, None, ws)
    dc.group_backward(dy, None, off, w, None, None, db1, ws)
    torch.cuda.synchronize()
    assert torch.equal(dx, dx1) and torch.equal(dw, dw1) and torch.equal(db, db1)


def test_group_without_rows():
    w, off = rand(3, 24, 16, seed=3, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int32, device="cuda")
    x, dy = torch.empty(0, 16, dtype=torch.bfloat16, device="cuda"), torch.empty(0, 24, dtype=torch.bfloat16, device="cuda")
    ws = torch.zeros(dc.group_workspace_bytes(0, 3, 16, 24, dc.BF16), dtype=torch.uint8, device="cuda")
    dc.group_forward(x, off, w, None, 0, dy, ws)
    dw, db = torch.full_like(w, 9.0), torch.full((3, 24), 9.0, device="cuda")
    dc.group_backward(dy, x, off, w, torch.empty_like(x), dw, db, ws)
    torch.cuda.synchronize()
    assert not bool(dw.any()) and not bool(db.any())


# runs: (rows, adapter); rows in front and behind without one; adapters, rank, c_in, c_out
ADAPTERS = [
    ([(1, 0)], 0, 1, 8, 8, 8),
    ([(1, 0)], 0, 1, 1, 1, 1),
    ([(1, 2), (1, 0), (1, -1), (1, 2)], 0, 3, 16, 256, 136),
    ([(1, i % 5) for i in range(64)], 0, 5, 16, 128, 264),
    ([(1, i % 7 - 1) for i in range(100)], 3, 6, 32, 200, 128),
    ([(2, 1), (3, 0), (0, 1), (40, 1), (5, 9)], 2, 2, 8, 64, 72),
    ([(300, 1), (1, 0), (17, -1), (129, 1)], 6, 2, 64, 136, 320),
    ([(128, 0), (128, 1), (256, 0)], 0, 2, 16, 512, 256),
    ([(61, 3), (70, 2)], 0, 4, 5, 96, 104),
    ([(33, 0), (120, 1)], 1, 2, 128, 72, 520),
    ([(20, 1), (90, 0)], 4, 2, 100, 131, 67),
    ([(1, 0), (1, 1)], 0, 2, 12, 33, 1001),
    ([], 9, 2, 16, 64, 64),
    ([], 400, 2, 16, 64, 200),
    ([(450, 0)], 0, 1, 48, 264, 1032),
    ([(2500, 0), (3, 1), (1300, 1), (200, -1)], 7, 2, 48, 1032, 2056),         # pairs of CTAs
    ([(1, 0)] * 30 + [(1900, 2), (1, 1), (1, -1), (1500, 0)], 3, 3, 16, 1100, 1032),
] + [([(k, (i + j) % 4 - (j % 7 == 3)) for j, k in enumerate(spread(rows, n, i))], 0, 4, r, c_in, c_out)
     for i, (rows, n, r, c_in, c_out) in enumerate(ADAPTER_FORMS)]


def adapter_inputs(case, dtype, shared=True):
    runs, tail, n, r, c_in, c_out = ADAPTERS[case]
    dt, rows = TYPES[dtype], sum(k for k, _ in runs) + tail
    x = rand(rows, c_in, seed=case + 11, dtype=dt)
    w = rand(c_out, c_in, seed=case + 12, dtype=dt, scale=1.0 / c_in ** 0.5) if shared else None
    a, b = rand(n, r, c_in, seed=case + 13, dtype=dt, scale=1.0 / c_in ** 0.5), rand(n, c_out, r, seed=case + 14, dtype=dt, scale=1.0 / r ** 0.5)
    scale = 0.25 + rand(n, seed=case + 15, dtype=torch.float32).abs()
    off = offsets_of([k for k, _ in runs])
    which = torch.tensor([k for _, k in runs], dtype=torch.int32, device="cuda")
    return x, w, a, b, scale, off, which


def keeps(dt):
    """Share of a term's magnitude that holding t (or u) may lose."""
    return 2.0 ** -16 if dt == torch.bfloat16 else 2.0 ** -24


def adapter_want(x, w, a, b, scale, off, which):
    """(y, slack) of the products and the adapters' part, in 64 bits; (t, its magnitudes) of every run with an adapter."""
    dt, rows, r = x.dtype, x.shape[0], a.shape[1]
    xd = x.double()
    y, s = torch.zeros(rows, b.shape[1], dtype=torch.float64, device="cuda"), torch.zeros(rows, b.shape[1], dtype=torch.float64, device="cuda")
    k = x.shape[1]
    if w is not None:
        y, s = xd @ w.double().t(), (xd.abs() @ w.double().abs().t()) * (k + r + 8) * U
    kept = []
    for (lo, hi), i in zip(runs_of(off), which.tolist()):
        if not 0 <= i < a.shape[0]:
            continue
        ad, bd, f = a[i].double(), b[i].double(), float(scale[i]) if scale is not None else 1.0
        t, m = f * (xd[lo:hi] @ ad.t()), f * (xd[lo:hi].abs() @ ad.abs().t())
        off_t = (k + 4) * U * m + keeps(dt) * t.abs()
        y[lo:hi] += t @ bd.t()
        s[lo:hi] += off_t @ bd.abs().t() + (k + 2 * r + 8) * U * (t.abs() @ bd.abs().t())
        kept.append((lo, hi, i, t, off_t))
    return y, s, kept


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("case", range(len(ADAPTERS)))
@pytest.mark.parametrize("form", ["plain", "all", "beside"])
def test_adapter_forward(form, case, dtype):
    x, w, a, b, scale, off, which = adapter_inputs(case, dtype, form != "beside")
    dt, rows, c_out = x.dtype, x.shape[0], b.shape[1]
    of_type(dt)
    want, slack, _ = adapter_want(x, w, a, b, scale if form != "plain" else None, off, which)
    bias = rand(c_out, seed=case, dtype=torch.float32) if form == "all" else None
    residual = rand(rows, c_out, seed=case + 1, dtype=dt) if form != "plain" else None
    if bias is not None:
        want, slack = want + bias.double(), slack + 4 * U * bias.double().abs()
    if residual is not None:
        want, slack = want + residual.double(), slack + 4 * U * (residual.double().abs() + want.abs())
    act = int(form == "all")
    ad = dc.Adapters(a, b, scale if form != "plain" else None)
    y, ws = Guarded(torch, (rows, c_out), dt, fill=float("nan")), workspace(dc.adapter_workspace_bytes(rows, ad.c_in, c_out, ad, ad.dtype))
    saved = Guarded(torch, (ad.saved(rows).numel(),), torch.uint8, fill=0xFF)
    if form == "beside":                         # in place
        y.t.copy_(residual)
        residual = y.t
    dc.adapter_forward(x, w, ad, off, which, bias, act, residual, saved.t, y.t, ws.t)
    torch.cuda.synchronize()
    y.check("y"), ws.check("workspace"), saved.check("saved")
    assert dc.workspace_status(ws.t) == dc.OK
    check(y.t, want.clamp(0, 6) if act else want, slack, "y")


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("case", range(len(ADAPTERS)))
@pytest.mark.parametrize("shared", [True, False])
def test_adapter_backward(shared, case, dtype):
    x, w, a, b, scale, off, which = adapter_inputs(case, dtype, shared)
    dt, rows, c_in, c_out, r = x.dtype, x.shape[0], x.shape[1], b.shape[1], a.shape[1]
    of_type(dt)
    dy = rand(rows, c_out, seed=case + 77, dtype=dt)
    ad = dc.Adapters(a, b, scale)
    ws, saved = workspace(dc.adapter_workspace_bytes(rows, c_in, c_out, ad, ad.dtype)), Guarded(torch, (ad.saved(rows).numel(),), torch.uint8, fill=0xFF)
    dc.adapter_forward(x, w, ad, off, which, None, 0, None, saved.t, torch.empty(rows, c_out, dtype=dt, device="cuda"), ws.t)
    ws.t[256:] = 0xFF                            # nothing is expected of it
    dx, da, db = Guarded(torch, (rows, c_in), dt, fill=float("nan")), Guarded(torch, tuple(a.shape), dt, fill=float("nan")), Guarded(torch, tuple(b.shape), dt, fill=float("nan"))
    dc.adapter_backward(dy, x, w, ad, off, which, saved.t, dx.t, da.t, db.t, ws.t)
    torch.cuda.synchronize()
    for g in (dx, da, db, ws, saved):
        g.check("adapter_backward")
    assert dc.workspace_status(ws.t) == dc.OK
    # dx is the forward formula of dy with the matrices turned round
    want, slack, back = adapter_want(dy, w.t().contiguous() if shared else None, b.transpose(1, 2).contiguous(), a.transpose(1, 2).contiguous(), scale, off, which)
    check(dx.t, want, slack, "dx")
    _, _, ahead = adapter_want(x, None, a, b, scale, off, which)
    da_want, da_slack = torch.zeros(a.shape, dtype=torch.float64, device="cuda"), torch.zeros(a.shape, dtype=torch.float64, device="cuda")
    db_want, db_slack = torch.zeros(b.shape, dtype=torch.float64, device="cuda"), torch.zeros(b.shape, dtype=torch.float64, device="cuda")
    for (lo, hi, i, t, off_t), (_, _, _, u, off_u) in zip(ahead, back):
        xs, ds = x[lo:hi].double(), dy[lo:hi].double()
        da_want[i] += u.t() @ xs
        da_slack[i] += off_u.t() @ xs.abs() + (rows + 8) * U * (u.abs().t() @ xs.abs())
        db_want[i] += ds.t() @ t
        db_slack[i] += ds.abs().t() @ off_t + (rows + 8) * U * (ds.abs().t() @ t.abs())
    check(da.t, da_want, da_slack, "da")
    check(db.t, db_want, db_slack, "db")


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("case", [4, 6, 15])
def test_adapter_backward_parts_alone(case, dtype):
    """Each set of gradients without the others gives the same bits, on workspaces that hold something else: what runs beside what, and waits for what, differs."""
    x, w, a, b, scale, off, which = adapter_inputs(case, dtype)
    dt, rows = x.dtype, x.shape[0]
    dy, ad = rand(rows, b.shape[1], seed=5, dtype=dt), dc.Adapters(a, b, scale)
    ws, saved = torch.zeros(dc.adapter_workspace_bytes(rows, ad.c_in, ad.c_out, ad, ad.dtype), dtype=torch.uint8, device="cuda"), ad.saved(rows)
    dc.adapter_forward(x, w, ad, off, which, None, 0, None, saved, torch.empty_like(dy), ws)
    outs = [torch.empty_like(x), torch.empty_like(a), torch.empty_like(b)]
    dc.adapter_backward(dy, x, w, ad, off, which, saved, *outs, ws)
    for wanted in ((0,), (1,), (2,), (0, 1), (0, 2), (1, 2)):
        for again in range(3):
            ws[256:] = 0xFF
            some = [torch.full_like(t, float("nan")) if k in wanted else None for k, t in enumerate(outs)]
            dc.adapter_backward(dy, x if 1 in wanted else None, w, ad, off, which, saved if 2 in wanted else None, *some, ws)
            for k in wanted:
                assert torch.equal(some[k], outs[k]), (wanted, k, again)


@pytest.mark.parametrize("dtype", list(TYPES))
def test_gradients_against_differences(dtype):
    """d/de of <forward(p + e v), dy> in 64 bits against <gradient, v>: the formula is linear in x, and in a and b apart."""
    x, w, a, b, scale, off, which = adapter_inputs(6, dtype)
    dt, rows, c_out = x.dtype, x.shape[0], b.shape[1]
    dy, ad = rand(rows, c_out, seed=5, dtype=dt), dc.Adapters(a, b, scale)
    ws, saved = torch.zeros(dc.adapter_workspace_bytes(rows, ad.c_in, c_out, ad, ad.dtype), dtype=torch.uint8, device="cuda"), ad.saved(rows)
    dc.adapter_forward(x, w, ad, off, which, None, 0, None, saved, torch.empty_like(dy), ws)
    dx, da, db = torch.empty_like(x), torch.empty_like(a), torch.empty_like(b)
    dc.adapter_backward(dy, x, w, ad, off, which, saved, dx, da, db, ws)
    torch.cuda.synchronize()

    def f(x, a, b):
        y = x @ w.double().t()
        for (lo, hi), i in zip(runs_of(off), which.tolist()):
            if i >= 0:
                y[lo:hi] += float(scale[i]) * (x[lo:hi] @ a[i].t()) @ b[i].t()
        return float((y * dy.double()).sum())

    p = [x.double(), a.double(), b.double()]
    for k, grad in enumerate((dx, da, db)):
        v = rand(*grad.shape, seed=40 + k, dtype=torch.float64)
        up, down = list(p), list(p)
        up[k], down[k] = p[k] + v, p[k] - v
        slope = (f(*up) - f(*down)) / 2
        # each element of the gradient is off by its rounding and a little; signs are random, the sum of all is a bound
        room = float((grad.double() * v).abs().sum()) * (half_step(dt) + 2.0 ** -15)
        assert abs(float((grad.double() * v).sum()) - slope) <= room, (k, slope, room)


# --------------------------------------------------------------------------- what masks leave out


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("runs", [[(1, i) for i in range(6)], [(3, 0), (60, 1), (5, 2), (1, 3), (200, 4), (7, 5)]])
def test_an_adapter_that_is_no_number_stays_in_its_rows(runs, dtype):
    """Infinities and NaN in one adapter, and in the rows of a request without one: other rows, and the gradients of other adapters, do not change."""
    dt, rows, c_in, c_out, r = TYPES[dtype], sum(k for k, _ in runs), 136, 264, 16
    x, w, dy = rand(rows, c_in, seed=1, dtype=dt), rand(c_out, c_in, seed=2, dtype=dt), rand(rows, c_out, seed=3, dtype=dt)
    a, b = rand(6, r, c_in, seed=4, dtype=dt), rand(6, c_out, r, seed=5, dtype=dt)
    off, which = offsets_of([k for k, _ in runs]), torch.tensor([k for _, k in runs], dtype=torch.int32, device="cuda")
    which[2] = -1
    lo, hi = runs_of(off)[2]
    ws = torch.zeros(dc.adapter_workspace_bytes(rows, c_in, c_out, dc.Adapters(a, b), dc.dtype_code(dt)), dtype=torch.uint8, device="cuda")

    def run(x, dy, a, b):
        ad = dc.Adapters(a, b)
        saved, y, dx, da, db = ad.saved(rows), torch.empty_like(dy), torch.empty_like(x), torch.empty_like(a), torch.empty_like(b)
        saved.fill_(0xFF)
        dc.adapter_forward(x, w, ad, off, which, None, 0, None, saved, y, ws)
        dc.adapter_backward(dy, x, w, ad, off, which, saved, dx, da, db, ws)
        torch.cuda.synchronize()
        assert dc.workspace_status(ws) == dc.OK
        return y, dx, da, db

    good = run(x, dy, a, b)
    a2, b2, x2, dy2 = a.clone(), b.clone(), x.clone(), dy.clone()
    a2[4, 3], b2[4, 7, 2], b2[4, 9] = float("nan"), float("inf"), float("-inf")
    a2[2], b2[2] = float("nan"), float("inf")     # an adapter that no run has
    x2[lo:hi], dy2[lo:hi] = float("nan"), float("inf")
    bad = run(x2, dy2, a2, b2)
    others = torch.ones(rows, dtype=torch.bool, device="cuda")
    others[lo:hi] = False
    for (p, q), i in zip(runs_of(off), which.tolist()):
        if i == 4:
            others[p:q] = False
    for k in (0, 1):
        assert torch.equal(good[k][others], bad[k][others]) and not bool(torch.isfinite(bad[k][lo:hi].float()).any())
    for k in (2, 3):
        assert torch.equal(good[k][[0, 1, 3, 5]], bad[k][[0, 1, 3, 5]]) and not bool(bad[k][2].any())
    p, q = runs_of(off)[4]
    assert bool((bad[0][p:q, 9].float().isnan() | bad[0][p:q, 9].float().isinf()).all())


def test_groups_beside_rows_that_are_no_numbers():
    """A group of NaN and infinities between two others: neither their results nor their gradients change."""
    for dt in TYPES.values():
        x, dy = rand(150, 72, seed=1, dtype=dt), rand(150, 264, seed=2, dtype=dt)
        w, off = rand(3, 264, 72, seed=3, dtype=dt), offsets_of([45, 30, 75])
        ws = torch.zeros(dc.group_workspace_bytes(150, 3, 72, 264, dc.dtype_code(dt)), dtype=torch.uint8, device="cuda")

        def run(x, dy):
            y, dx, dw, db = torch.empty_like(dy), torch.empty_like(x), torch.empty_like(w), torch.empty(3, 264, device="cuda")
            dc.group_forward(x, off, w, None, 0, y, ws)
            dc.group_backward(dy, x, off, w, dx, dw, db, ws)
            torch.cuda.synchronize()
            return y, dx, dw, db

        good = run(x, dy)
        x[45:75], dy[45:75] = float("nan"), float("-inf")
        bad = run(x, dy)
        for k in (0, 1):
            assert torch.equal(good[k][:45], bad[k][:45]) and torch.equal(good[k][75:], bad[k][75:])
        for k in (2, 3):
            assert torch.equal(good[k][[0, 2]], bad[k][[0, 2]])
        assert bool(bad[3][1].isinf().all()) and bool(bad[0][45:75].isnan().all())


def test_fp32_results_that_are_no_numbers():
    """fp32 products go by terms of bf16, of which an infinity has none: what comes out is what FMAs give, in all three products and of few rows and many."""
    for sizes, c_in, c_out in (([3, 2], 72, 40), ([200, 90], 200, 136)):
        rows = sum(sizes)
        x, dy = rand(rows, c_in, seed=1, dtype=torch.float32), rand(rows, c_out, seed=2, dtype=torch.float32)
        w, off = rand(2, c_out, c_in, seed=3, dtype=torch.float32), offsets_of(sizes)
        x[0, 5], x[1, 7], x[sizes[0], 3] = float("inf"), float("nan"), 3.4e38
        dy[0, 2], dy[2, 1] = float("-inf"), float("inf")
        w[0, 4, 5], w[1, 1, 3] = 0.0, 0.5
        ws = torch.zeros(dc.group_workspace_bytes(rows, 2, c_in, c_out, dc.F32), dtype=torch.uint8, device="cuda")
        y, dx, dw, db = torch.empty_like(dy), torch.empty_like(x), torch.empty_like(w), torch.empty(2, c_out, device="cuda")
        dc.group_forward(x, off, w, None, 0, y, ws)
        dc.group_backward(dy, x, off, w, dx, dw, db, ws)
        torch.cuda.synchronize()
        assert dc.workspace_status(ws) == dc.OK
        for g, (lo, hi) in enumerate(runs_of(off)):
            a, b, m = x[lo:hi].double(), dy[lo:hi].double(), w[g].double()
            for got, p, q in ((y[lo:hi], a, m.t()), (dx[lo:hi], b, m), (dw[g], b.t(), a), (db[g][:, None], b.t(), torch.ones(hi - lo, 1, dtype=torch.float64, device="cuda"))):
                want = (p[:, :, None] * q[None]).sum(1).float()      # element by element: a library product may skip a NaN
                assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.isinf(), want.isinf())
                fine = want.isfinite()
                assert torch.equal(torch.sign(got[~fine]).nan_to_num(), torch.sign(want[~fine]).nan_to_num())
                assert bool(((got - want)[fine].abs() <= 1e-4 * want[fine].abs() + 1e-3).all())


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows", [1, 20, 400])
def test_what_rows_keep_up_to_the_largest_number(rows, dtype):
    """t beyond the largest bf16, where its first term alone would be an infinity: a number still, and so is what is made of it."""
    dt = TYPES[dtype]
    of_type(dt)
    for sign in (1.0, -1.0):
        x = torch.zeros(rows, 64, dtype=dt, device="cuda")
        x[:, 0], x[:, 1] = sign * 2.0 ** 127, sign * 127.0 / 128 * 2.0 ** 127
        x[:, 2] = sign * 0.75 * 2.0 ** 120       # together (2 - 2^-7 + 0.75 2^-7) 2^127: beyond (2 - 2^-7) 2^127, in fp32's range
        a, b = torch.zeros(1, 4, 64, dtype=dt, device="cuda"), torch.zeros(1, 72, 4, dtype=dt, device="cuda")
        a[0, 0, :3], b[0, :, 0] = 1.0, 2.0 ** -20
        ad, off, which = dc.Adapters(a, b), offsets_of([rows]), torch.zeros(1, dtype=torch.int32, device="cuda")
        y, ws = Guarded(torch, (rows, 72), dt, fill=0), workspace(dc.adapter_workspace_bytes(rows, 64, 72, ad, ad.dtype))
        saved = ad.saved(rows)
        dc.adapter_forward(x, None, ad, off, which, None, 0, None, saved, y.t, ws.t)
        db = torch.empty_like(b)
        dy = torch.full((rows, 72), 2.0 ** -20 / rows, dtype=dt, device="cuda")
        dc.adapter_backward(dy, None, None, ad, off, which, saved, None, None, db, ws.t)
        torch.cuda.synchronize()
        want, slack, _ = adapter_want(x, None, a, b, None, off, which)
        check(y.t, want, slack, "y")
        t = (x.double() @ a[0].double().t())
        check(db[0], dy.double().t() @ t, (keeps(dt) + (rows + 70) * U) * (dy.double().abs().t() @ t.abs()), "db")


def test_offsets_out_of_order_stay_inside():
    """What such offsets give is undefined, but inside the arrays."""
    for dt in TYPES.values():
        for numbers in ([0, 900, 3, 12], [-5, 4, 2, 7], [7, 7, 7, 7], [12, 10, 5, 0], [2 ** 31 - 1, -2 ** 31, 9, 11], [3, 9, 10 ** 9, 6]):
            off = torch.tensor(numbers, dtype=torch.int32, device="cuda")
            x, dy = rand(11, 40, seed=1, dtype=dt), rand(11, 72, seed=2, dtype=dt)
            w = rand(3, 72, 40, seed=3, dtype=dt)
            g = [Guarded(torch, s, t, fill=0) for s, t in (((11, 72), dt), ((11, 40), dt), ((3, 72, 40), dt), ((3, 72), torch.float32))]
            ws = workspace(dc.group_workspace_bytes(11, 3, 40, 72, dc.dtype_code(dt)))
            dc.group_forward(x, off, w, None, 0, g[0].t, ws.t)
            dc.group_backward(dy, x, off, w, g[1].t, g[2].t, g[3].t, ws.t)
            a, b = rand(2, 8, 40, seed=4, dtype=dt), rand(2, 72, 8, seed=5, dtype=dt)
            ad, which = dc.Adapters(a, b), torch.tensor([1, 77, -3], dtype=torch.int32, device="cuda")
            ws2, saved = workspace(dc.adapter_workspace_bytes(11, 40, 72, ad, ad.dtype)), Guarded(torch, (ad.saved(11).numel(),), torch.uint8, fill=0)
            da, db = Guarded(torch, (2, 8, 40), dt, fill=0), Guarded(torch, (2, 72, 8), dt, fill=0)
            dc.adapter_forward(x, w[0].contiguous(), ad, off, which, None, 0, None, saved.t, g[0].t, ws2.t)
            dc.adapter_backward(dy, x, w[0].contiguous(), ad, off, which, saved.t, g[1].t, da.t, db.t, ws2.t)
            torch.cuda.synchronize()
            for q in g + [ws, ws2, saved, da, db]:
                q.check(str(numbers))
            assert dc.workspace_status(ws.t) == dc.OK and dc.workspace_status(ws2.t) == dc.OK


# --------------------------------------------------------------------------- streams, graphs, sizes


class Step:
    """A training step of two adapters beside a shared matrix, and of groups behind it, on buffers of its own."""

    def __init__(self, seed, dt=torch.bfloat16, rows=700):
        self.off, self.which = offsets_of([rows // 2, 1, rows - rows // 2 - 1]), torch.tensor([0, 1, 1], dtype=torch.int32, device="cuda")
        self.goff = offsets_of([rows // 3, 0, rows - rows // 3])
        self.w, self.wg = rand(256, 200, seed=1, dtype=dt, scale=0.1), rand(3, 136, 256, seed=2, dtype=dt, scale=0.1)
        self.ad = dc.Adapters(rand(2, 16, 200, seed=3, dtype=dt, scale=0.1), rand(2, 256, 16, seed=4, dtype=dt))
        self.x, self.dz = torch.empty(rows, 200, dtype=dt, device="cuda"), torch.empty(rows, 136, dtype=dt, device="cuda")
        self.fill(seed)
        self.saved, self.y, self.z = self.ad.saved(rows), torch.empty(rows, 256, dtype=dt, device="cuda"), torch.empty_like(self.dz)
        self.dy, self.dx, self.dwg = torch.empty_like(self.y), torch.empty_like(self.x), torch.empty_like(self.wg)
        self.da, self.db, self.dbg = torch.empty_like(self.ad.a), torch.empty_like(self.ad.b), torch.empty(3, 136, device="cuda")
        size = max(dc.adapter_workspace_bytes(rows, 200, 256, self.ad, self.ad.dtype), dc.group_workspace_bytes(rows, 3, 256, 136, self.ad.dtype))
        self.ws = torch.zeros(size, dtype=torch.uint8, device="cuda")

    def fill(self, seed):
        self.x.copy_(rand(*self.x.shape, seed=seed, dtype=torch.float32)), self.dz.copy_(rand(*self.dz.shape, seed=seed + 1, dtype=torch.float32))

    def __call__(self, stream=None):
        dc.adapter_forward(self.x, self.w, self.ad, self.off, self.which, None, 0, None, self.saved, self.y, self.ws, stream)
        dc.group_forward(self.y, self.goff, self.wg, None, 0, self.z, self.ws, stream)
        dc.group_backward(self.dz, self.y, self.goff, self.wg, self.dy, self.dwg, self.dbg, self.ws, stream)
        dc.adapter_backward(self.dy, self.x, self.w, self.ad, self.off, self.which, self.saved, self.dx, self.da, self.db, self.ws, stream)

    def outputs(self):
        torch.cuda.synchronize()
        assert dc.workspace_status(self.ws) == dc.OK
        return [t.clone() for t in (self.y, self.z, self.dy, self.dwg, self.dbg, self.dx, self.da, self.db)]


@pytest.mark.parametrize("rows", [30, 700])
@pytest.mark.parametrize("dtype", list(TYPES))
def test_a_step_repeats_itself_and_in_a_graph(dtype, rows):
    """The same bits every time, alone, on another stream, and replayed from a graph with other inputs than it was captured with."""
    step = Step(5, TYPES[dtype], rows)
    step()
    first = step.outputs()
    for _ in range(20):
        step()
    assert all(torch.equal(a, b) for a, b in zip(first, step.outputs()))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    step(side)
    assert all(torch.equal(a, b) for a, b in zip(first, step.outputs()))
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            for _ in range(3):
                step()
    step.fill(77)
    torch.cuda.synchronize()
    step()
    other = step.outputs()
    step.fill(5)
    graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(first, step.outputs()))
    step.fill(77)
    for _ in range(5):
        graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(other, step.outputs()))
    assert not all(torch.equal(a, b) for a, b in zip(first, other))


def test_steps_on_two_streams_at_once():
    steps, streams = [Step(5), Step(9)], [torch.cuda.Stream(), torch.cuda.Stream()]
    want = []
    for s in steps:
        s()
        want.append(s.outputs())
    for _ in range(30):
        for s, st in zip(steps, streams):
            s(st)
    for s, w in zip(steps, want):
        assert all(torch.equal(a, b) for a, b in zip(w, s.outputs()))


def test_a_step_follows_what_writes_its_inputs():
    """Calls right behind kernels of other libraries that write what they read, and in front of such that read what they write."""
    step = Step(5)
    step()
    want = step.outputs()
    x, dz = step.x.clone(), step.dz.clone()
    total = None
    for _ in range(30):
        step.x.zero_(), step.dz.zero_(), step.y.fill_(3.0), step.saved.fill_(0xFF)
        step.x.copy_(x), step.dz.copy_(dz)
        step()
        s = step.dx.double().sum() + step.da.double().sum() + step.dwg.double().sum()
        total = s if total is None else torch.stack((total, s)).max()
        assert bool(total == s)
    assert all(torch.equal(a, b) for a, b in zip(want, step.outputs()))


def test_beside_a_projection_in_4_bits():
    """A layer whose own weights are held in 4 bits, with adapters added in place, in front of experts: each stage from what the one before gave."""
    dt, rows, c_in, c_out = torch.bfloat16, 133, 256, 512
    of_type(dt)
    x, w = rand(rows, c_in, seed=1, dtype=dt), rand(c_out, c_in, seed=2, dtype=torch.float32, scale=c_in ** -0.5)
    q = dc.Q4Matrix(c_out, c_in, dc.NV4, dc.q4_tensor_scale(float(w.abs().max())))
    dc.q4_quantize(w, q)
    y = torch.empty(rows, c_out, dtype=dt, device="cuda")
    qws = torch.zeros(dc.q4_workspace_bytes(rows, c_in, dc.NV4), dtype=torch.uint8, device="cuda")
    dc.q4_forward(x, q, dc.q4_tensor_scale(float(x.abs().max())), None, 0, None, y, qws)
    base = y.clone()
    a, b = rand(3, 16, c_in, seed=3, dtype=dt, scale=c_in ** -0.5), rand(3, c_out, 16, seed=4, dtype=dt, scale=0.25)
    ad, off, which = dc.Adapters(a, b), offsets_of([1, 100, 2, 30]), torch.tensor([2, 0, -1, 1], dtype=torch.int32, device="cuda")
    ws = torch.zeros(dc.adapter_workspace_bytes(rows, c_in, c_out, ad, dc.BF16), dtype=torch.uint8, device="cuda")
    dc.adapter_forward(x, None, ad, off, which, None, dc.ACT_RELU6, y, ad.saved(rows), y, ws)
    want, slack, _ = adapter_want(x, None, a, b, None, off, which)
    want, slack = want + base.double(), slack + 4 * U * (base.double().abs() + want.abs())
    check(y, want.clamp(0, 6), slack, "beside 4 bits")
    experts, goff, z = rand(2, 136, c_out, seed=6, dtype=dt, scale=c_out ** -0.5), offsets_of([60, 73]), torch.empty(rows, 136, dtype=dt, device="cuda")
    dc.group_forward(y, goff, experts, None, 0, z, torch.zeros(dc.group_workspace_bytes(rows, 2, c_out, 136, dc.BF16), dtype=torch.uint8, device="cuda"))
    want, slack, _ = group_want(y, goff, experts, None, 0)
    check(z, want, slack, "experts")


def test_arrays_beyond_32_bits():
    """x, y and the matrices each with more than 2^32 elements; rows, groups and adapters behind that."""
    dt = torch.bfloat16
    of_type(dt)
    free = torch.cuda.mem_get_info()[0]
    if free < 60 << 30:
        pytest.skip("not enough memory")
    rows, c = (1 << 20) + 70000, 4096            # 4.6e9 elements
    x = torch.zeros(rows, c, dtype=dt, device="cuda")
    x[-300:] = rand(300, c, seed=1, dtype=dt)
    w = rand(2, 64, c, seed=2, dtype=dt, scale=c ** -0.5)
    off = torch.tensor([0, rows - 300, rows], dtype=torch.int32, device="cuda")
    y, ws = torch.empty(rows, 64, dtype=dt, device="cuda"), torch.zeros(dc.group_workspace_bytes(rows, 2, c, 64, dc.BF16), dtype=torch.uint8, device="cuda")
    dc.group_forward(x, off, w, None, 0, y, ws)
    want, slack, _ = group_want(x[-300:], offsets_of([0, 300]), w, None, 0)
    check(y[-300:], want, slack, "x beyond 32 bits")
    assert not bool(y[:-300].any())
    dw = torch.empty_like(w)
    dc.group_backward(y, x, off, w, None, dw, None, ws)
    a, b = y[-300:].double(), x[-300:].double()
    check(dw[1], a.t() @ b, 304 * U * (a.abs().t() @ b.abs()), "dw")
    assert not bool(dw[0].any())
    back = rand(2, c, 64, seed=9, dtype=dt, scale=0.125)                 # and y beyond 32 bits
    dc.group_forward(y, off, back, None, 0, x, torch.zeros(dc.group_workspace_bytes(rows, 2, 64, c, dc.BF16), dtype=torch.uint8, device="cuda"))
    want, slack, _ = group_want(y[-300:], offsets_of([0, 300]), back, None, 0)
    check(x[-300:], want, slack, "y beyond 32 bits")
    del x, y
    groups = 260                                  # 4.4e9 elements of matrices
    w = torch.zeros(groups, c, c, dtype=dt, device="cuda")
    w[-1] = rand(c, c, seed=3, dtype=dt, scale=c ** -0.5)
    for n in (3, 200):
        x, y = rand(n, c, seed=4, dtype=dt), torch.empty(n, c, dtype=dt, device="cuda")
        off = torch.zeros(groups + 1, dtype=torch.int32, device="cuda")
        off[-1] = n
        ws = torch.zeros(dc.group_workspace_bytes(n, groups, c, c, dc.BF16), dtype=torch.uint8, device="cuda")
        dc.group_forward(x, off, w, None, 0, y, ws)
        want, slack, _ = group_want(x, offsets_of([n]), w[-1:], None, 0)
        check(y, want, slack, "matrices beyond 32 bits")
        dw = torch.full_like(w, 5.0)
        dc.group_backward(y, x, off, w, None, dw, None, ws)
        a, b = y.double(), x.double()
        check(dw[-1], a.t() @ b, (n + 4) * U * (a.abs().t() @ b.abs()), "dw")
        assert not bool(dw[:-1].any())
        del dw


def test_fp32_matrices_beyond_32_bits():
    """Read as they lie."""
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("not enough memory")
    dt, groups, n, c = torch.float32, 260, 3, 4096
    of_type(dt)
    w = torch.zeros(groups, c, c, device="cuda")
    w[-1] = rand(c, c, seed=3, dtype=dt, scale=c ** -0.5)
    x, dy = rand(n, c, seed=4, dtype=dt), rand(n, c, seed=5, dtype=dt)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    off = torch.zeros(groups + 1, dtype=torch.int32, device="cuda")
    off[-1] = n
    assert dc.group_plan(n, groups, c, c, 0, dc.F32, dc.GROUP_FORWARD).form == dc.GROUP_FMAS
    ws = torch.empty(dc.group_workspace_bytes(n, groups, c, c, dc.F32), dtype=torch.uint8, device="cuda")
    ws[:256] = 0
    dc.group_forward(x, off, w, None, 0, y, ws)
    dc.group_backward(dy, None, off, w, dx, None, None, ws)
    wd = w[-1].double()
    check(y, x.double() @ wd.t(), (c + 4) * U * (x.double().abs() @ wd.abs().t()), "y")
    check(dx, dy.double() @ wd, (c + 4) * U * (dy.double().abs() @ wd.abs()), "dx")


def test_tensors_of_the_host_are_refused():
    step = Step(5)
    with pytest.raises(ValueError):
        dc.group_forward(step.y, step.goff.cpu(), step.wg, None, 0, step.z, step.ws)
    with pytest.raises(ValueError):
        dc.group_backward(step.dz, step.y.cpu(), step.goff, step.wg, step.dy, step.dwg, None, step.ws)
    with pytest.raises(ValueError):
        dc.adapter_forward(step.x, step.w, step.ad, step.off, step.which.cpu(), None, 0, None, step.saved, step.y, step.ws)
    with pytest.raises(ValueError):
        dc.adapter_backward(step.dy, step.x, step.w, step.ad, step.off, step.which, step.saved.cpu(), step.dx, step.da, step.db, step.ws)


def test_without_the_native_marshalling(monkeypatch):
    step = Step(5)
    step()
    want = step.outputs()
    dc.lib()
    monkeypatch.setattr(dc, "_native", dc._NoNative)
    step.y.zero_(), step.da.zero_(), step.dwg.zero_()
    step()
    assert all(torch.equal(a, b) for a, b in zip(want, step.outputs()))

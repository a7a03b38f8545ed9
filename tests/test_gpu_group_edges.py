"""Grouped products and adapters on the GPU: gradients of which a CTA makes several tiles, infinities, rows in front of the first run.

Tolerances as in test_gpu_group.py.  What a bf16 row keeps of an adapter, t, is two terms of its sign: the first t cut off to 8 bits, which leaves r < 2^-7 of t's leading
bit, the second r rounded to 8 bits, half a last place of it at most 2^-9 of 2^-7: 2^-16 of t.  Where r is 0 the first is a step less, and r that step, which is exact."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2301_12187_b200 import dc
from tests.group_sizes import spread
from tests.parity_util import Guarded
from tests.test_gpu_group import TYPES, U, adapter_want, check, group_want, of_type, offsets_of, rand, workspace


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rank", [1, 8, 16, 17, 48, 80, 112, 128])
def test_more_tiles_of_gradients_than_ctas(rank, dtype):
    """64 adapters, of which 13 are named by no run, of 1024 -> 1160: 512 and 640 tiles of gradients, more than three to an SM, of runs that end inside pieces."""
    dt, n, c_in, c_out, rows = TYPES[dtype], 64, 1024, 1160, 700
    of_type(dt)
    sizes = spread(rows, 90, rank)
    off = offsets_of(sizes)
    which = torch.tensor([(i * 7) % n if (i * 7) % 3 else -1 for i in range(len(sizes))], dtype=torch.int32, device="cuda")
    x, dy = rand(rows, c_in, seed=1, dtype=dt), rand(rows, c_out, seed=2, dtype=dt)
    a, b = rand(n, rank, c_in, seed=3, dtype=dt, scale=c_in ** -0.5), rand(n, c_out, rank, seed=4, dtype=dt, scale=rank ** -0.5)
    scale = 0.25 + rand(n, seed=5, dtype=torch.float32).abs()
    ad = dc.Adapters(a, b, scale)
    ws, saved = workspace(dc.adapter_workspace_bytes(rows, c_in, c_out, ad, ad.dtype)), Guarded(torch, (ad.saved(rows).numel(),), torch.uint8, fill=0xFF)
    dc.adapter_forward(x, None, ad, off, which, None, 0, None, saved.t, torch.empty_like(dy), ws.t)
    da, db = Guarded(torch, tuple(a.shape), dt, fill=float("nan")), Guarded(torch, tuple(b.shape), dt, fill=float("nan"))
    dc.adapter_backward(dy, x, None, ad, off, which, saved.t, None, da.t, db.t, ws.t)
    torch.cuda.synchronize()
    for g in (da, db, ws, saved):
        g.check("gradients")
    assert dc.workspace_status(ws.t) == dc.OK
    _, _, ahead = adapter_want(x, None, a, b, scale, off, which)
    _, _, back = adapter_want(dy, None, b.transpose(1, 2).contiguous(), a.transpose(1, 2).contiguous(), scale, off, which)
    zeros = [torch.zeros(t.shape, dtype=torch.float64, device="cuda") for t in (a, a, b, b)]
    da_want, da_slack, db_want, db_slack = zeros
    for (lo, hi, i, t, off_t), (_, _, _, u, off_u) in zip(ahead, back):
        xs, ds = x[lo:hi].double(), dy[lo:hi].double()
        da_want[i] += u.t() @ xs
        da_slack[i] += off_u.t() @ xs.abs() + (rows + 8) * U * (u.abs().t() @ xs.abs())
        db_want[i] += ds.t() @ t
        db_slack[i] += ds.abs().t() @ off_t + (rows + 8) * U * (ds.abs().t() @ t.abs())
    check(da.t, da_want, da_slack, "da")
    check(db.t, db_want, db_slack, "db")
    without = sorted(set(range(n)) - {i for _, _, i, _, _ in ahead})
    assert len(without) == 13 and not bool(da.t[without].any()) and not bool(db.t[without].any())


def test_an_infinity_among_many_rows():
    """fp32 gradients of a group of two million rows with infinities in dy and in x: what it makes of a gradient is worked out again by FMAs, over all rows, and comes
    in the time that the waits for it allow."""
    dt, rows, c_in, c_out = torch.float32, 1 << 21, 72, 136
    of_type(dt)
    x, dy = rand(rows, c_in, seed=1, dtype=dt), rand(rows, c_out, seed=2, dtype=dt)
    off, w = offsets_of([rows]), torch.empty(1, c_out, c_in, device="cuda")
    ws = torch.zeros(dc.group_workspace_bytes(rows, 1, c_in, c_out, dc.F32), dtype=torch.uint8, device="cuda")
    a, b = dy.double(), x.double()
    want, slack = a.t() @ b, (rows + 4) * U * (a.abs().t() @ b.abs())
    sums, room = a.sum(0), (rows + 4) * U * a.abs().sum(0)
    for r, i, value in ((rows // 2 + 11, 77, float("inf")), (rows - 3, 5, float("-inf"))):
        want[i], sums[i] = torch.sign(b[r]) * value, value
        dy[r, i] = value
    keep = want[[77, 5], 40].clone()
    want[:, 40] = torch.sign(a[17]) * float("inf")
    want[[77, 5], 40] += keep                    # of the other sign: no number
    x[17, 40] = float("inf")
    dw, db = Guarded(torch, (1, c_out, c_in), dt, fill=7.0), Guarded(torch, (1, c_out), dt, fill=7.0)
    dc.group_backward(dy, x, off, w, None, dw.t, db.t, ws)
    torch.cuda.synchronize()
    dw.check("dw"), db.check("db")
    assert dc.workspace_status(ws) == dc.OK
    got = dw.t[0].double()
    fine = want.isfinite()
    assert torch.equal(got[~fine].nan_to_num(), want[~fine].nan_to_num()) and torch.equal(got.isnan(), want.isnan())
    check(torch.where(fine, got, 0.0).float(), torch.where(fine, want, 0.0), slack, "dw")
    assert torch.equal(db.t[0][[77, 5]].double(), sums[[77, 5]])
    fine = sums.isfinite()
    assert bool(((db.t[0].double() - sums).abs()[fine] <= room[fine]).all())


def each_by_each(p, q):
    """p [m, k] times q [k, n] in 64 bits, element by element: a library product may skip a NaN."""
    out = [(p[i:i + 16, :, None].double() * q[None].double()).sum(1) for i in range(0, p.shape[0], 16)]
    return torch.cat(out)


def finite_part(*tensors):
    return [torch.where(t.isfinite(), t, torch.zeros_like(t)) for t in tensors]


def check_class(got, want, slack, what):
    got = got.double()
    assert torch.equal(got.isnan(), want.isnan()), "%s: NaN in %d places, not %d" % (what, int(got.isnan().sum()), int(want.isnan().sum()))
    far = want.isinf()
    assert torch.equal(got.isinf(), far) and torch.equal(got[far], want[far]), "%s: infinities" % what
    fine = want.isfinite()
    check(torch.where(fine, got, 0.0).float(), torch.where(fine, want, 0.0), slack, what)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rank", [8, 48])
@pytest.mark.parametrize("sizes", [[1, 1, 1, 1], [20, 1, 8, 31], [150, 3, 100, 147]])
@pytest.mark.parametrize("shared", [True, False])
def test_infinities_are_what_the_formula_makes_of_them(shared, sizes, rank, dtype):
    """Infinities in an adapter's matrices, in x and in dy: infinities, and NaN where infinities cancel, in y, dx, da and db, whichever way rows go.  What a row keeps
    of its adapter may lie on a bf16 number, so that its low terms are 0, or between two."""
    dt, rows, c_in, c_out = TYPES[dtype], sum(sizes), 136, 264
    of_type(dt)
    x, dy, w = rand(rows, c_in, seed=1, dtype=dt), rand(rows, c_out, seed=2, dtype=dt), rand(c_out, c_in, seed=3, dtype=dt) if shared else None
    a, b = rand(4, rank, c_in, seed=4, dtype=dt), rand(4, c_out, rank, seed=5, dtype=dt)
    off, which = offsets_of(sizes), torch.arange(4, dtype=torch.int32, device="cuda")
    runs = list(zip(off.tolist()[:-1], off.tolist()[1:]))
    x[0], dy[0] = 0.0, 0.0
    x[0, 0] = dy[0, 0] = 1.0                     # t and u are a column of the adapter's
    b[0, 5, 2], b[0, 6, 1], b[0, 7, :2] = float("inf"), float("-inf"), float("inf")
    a[0, 1, 9], a[0, 2, 10], a[1, 3, 4] = float("inf"), float("-inf"), float("inf")
    x[runs[2][0], 9], dy[runs[3][1] - 1, 11] = float("inf"), float("-inf")
    ad = dc.Adapters(a, b)
    ws, saved = workspace(dc.adapter_workspace_bytes(rows, c_in, c_out, ad, ad.dtype)), ad.saved(rows)
    y, y6 = torch.empty_like(dy), torch.empty_like(dy)
    dx, da, db = torch.empty_like(x), torch.empty_like(a), torch.empty_like(b)
    dc.adapter_forward(x, w, ad, off, which, None, dc.ACT_RELU6, None, saved, y6, ws.t)
    dc.adapter_forward(x, w, ad, off, which, None, 0, None, saved, y, ws.t)
    dc.adapter_backward(dy, x, w, ad, off, which, saved, dx, da, db, ws.t)
    torch.cuda.synchronize()
    assert dc.workspace_status(ws.t) == dc.OK
    ws.check("workspace")
    y_want, dx_want = torch.zeros(rows, c_out, dtype=torch.float64, device="cuda"), torch.zeros(rows, c_in, dtype=torch.float64, device="cuda")
    if shared:
        y_want, dx_want = each_by_each(x, w.t()), each_by_each(dy, w)
    da_want, db_want = a.double(), b.double()
    fx, fdy, fa, fb = finite_part(x, dy, a, b)
    _, y_slack, ahead = adapter_want(fx, w, fa, fb, None, off, which)
    _, dx_slack, back = adapter_want(fdy, w.t().contiguous() if shared else None, fb.transpose(1, 2).contiguous(), fa.transpose(1, 2).contiguous(), None, off, which)
    da_slack, db_slack = torch.zeros_like(da_want), torch.zeros_like(db_want)
    for i, (lo, hi) in enumerate(runs):
        t, u = each_by_each(x[lo:hi], a[i].t()), each_by_each(dy[lo:hi], b[i])
        y_want[lo:hi] += each_by_each(t, b[i].t())
        dx_want[lo:hi] += each_by_each(u, a[i])
        da_want[i], db_want[i] = each_by_each(u.t(), x[lo:hi]), each_by_each(dy[lo:hi].t(), t)
        (_, _, _, t, off_t), (_, _, _, u, off_u) = ahead[i], back[i]
        xs, ds = fx[lo:hi].double(), fdy[lo:hi].double()
        da_slack[i] = off_u.t() @ xs.abs() + (rows + 8) * U * (u.abs().t() @ xs.abs())
        db_slack[i] = ds.abs().t() @ off_t + (rows + 8) * U * (ds.abs().t() @ t.abs())
    assert all(bool(t.isinf().any()) and bool(t.isnan().any()) for t in (y_want, dx_want)) and all(bool(t.isinf().any()) for t in (da_want, db_want))
    check_class(y, y_want, y_slack, "y")
    check_class(dx, dx_want, dx_slack, "dx")
    check_class(da, da_want, da_slack, "da")
    check_class(db, db_want, db_slack, "db")
    check_class(y6, torch.where(y_want.isnan(), 0.0, y_want.clamp(0, 6)), y_slack, "y under ReLU6")      # a NaN is 0 there, as in all of the library


def test_those_sizes_take_both_ways():
    """The sizes above go by short runs and by tiles."""
    forms = {dc.group_plan(n, 4, 136, 264, 8, dc.BF16, dc.GROUP_FORWARD).form for n in (4, 60, 400)}
    assert {dc.GROUP_FEW_ROWS, dc.GROUP_TILES} <= forms


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("front,sizes,c_in,c_out", [(1, [1, 2], 72, 40), (5, [3, 0, 2], 136, 264), (70, [30, 0, 100], 72, 136), (129, [300, 1, 270], 520, 264),
                                                     (3, [1] * 40, 264, 1032)])
def test_rows_in_front_of_the_first_run(front, sizes, c_in, c_out, dtype):
    """The first offset above 0: rows in front of it belong to no group, and stay as they were; to no adapter's run, and go without.  They hold NaN where nothing may read them."""
    dt, n, rows = TYPES[dtype], len(sizes), front + sum(sizes) + 4
    of_type(dt)
    off = (offsets_of(sizes) + front).int()
    lo, hi = front, rows - 4
    x, dy = rand(rows, c_in, seed=1, dtype=dt), rand(rows, c_out, seed=2, dtype=dt)
    w = rand(n, c_out, c_in, seed=3, dtype=dt)
    xn, dyn = x.clone(), dy.clone()
    for t in (xn, dyn):
        t[:lo], t[hi:] = float("nan"), float("inf")
    ws = workspace(dc.group_workspace_bytes(rows, n, c_in, c_out, dc.dtype_code(dt)))
    y, dx, dw = Guarded(torch, (rows, c_out), dt, fill=7.0), Guarded(torch, (rows, c_in), dt, fill=7.0), Guarded(torch, (n, c_out, c_in), dt, fill=7.0)
    db = Guarded(torch, (n, c_out), torch.float32, fill=7.0)
    dc.group_forward(xn, off, w, None, 0, y.t, ws.t)
    dc.group_backward(dyn, xn, off, w, dx.t, dw.t, db.t, ws.t)
    torch.cuda.synchronize()
    for q in (y, dx, dw, db, ws):
        q.check("groups")
    want, slack, mine = group_want(x, off, w, None, 0)
    check(y.t[mine], want[mine], slack[mine], "y")
    assert bool((y.t[~mine] == 7.0).all()) and bool((dx.t[~mine] == 7.0).all()) and int(mine.sum()) == hi - lo
    for g, (p, q) in enumerate(zip(off.tolist()[:-1], off.tolist()[1:])):
        a, b, m = dy[p:q].double(), x[p:q].double(), w[g].double()
        check(dx.t[p:q], a @ m, (c_out + 4) * U * (a.abs() @ m.abs()), "dx")
        check(dw.t[g], a.t() @ b, (q - p + 4) * U * (a.abs().t() @ b.abs()), "dw")
        assert bool(((db.t[g].double() - a.sum(0)).abs() <= (q - p + 4) * U * a.abs().sum(0)).all())
    # adapters
    a, b, shared = rand(n, 16, c_in, seed=4, dtype=dt), rand(n, c_out, 16, seed=5, dtype=dt), w[0].contiguous()
    ad, which = dc.Adapters(a, b), torch.arange(n, dtype=torch.int32, device="cuda")
    ws, saved = workspace(dc.adapter_workspace_bytes(rows, c_in, c_out, ad, ad.dtype)), Guarded(torch, (ad.saved(rows).numel(),), torch.uint8, fill=0xFF)
    da, db = Guarded(torch, tuple(a.shape), dt, fill=7.0), Guarded(torch, tuple(b.shape), dt, fill=7.0)
    dc.adapter_forward(x, shared, ad, off, which, None, 0, None, saved.t, y.t, ws.t)
    dc.adapter_backward(dy, x, shared, ad, off, which, saved.t, dx.t, da.t, db.t, ws.t)
    torch.cuda.synchronize()
    for q in (y, dx, da, db, ws, saved):
        q.check("adapters")
    want, slack, ahead = adapter_want(x, shared, a, b, None, off, which)
    check(y.t, want, slack, "y of adapters")
    want, slack, back = adapter_want(dy, shared.t().contiguous(), b.transpose(1, 2).contiguous(), a.transpose(1, 2).contiguous(), None, off, which)
    check(dx.t, want, slack, "dx of adapters")
    da_first, db_first = da.t.clone(), db.t.clone()
    dc.adapter_forward(xn, shared, ad, off, which, None, 0, None, saved.t, y.t, ws.t)
    dc.adapter_backward(dyn, xn, shared, ad, off, which, saved.t, dx.t, da.t, db.t, ws.t)
    torch.cuda.synchronize()
    assert torch.equal(da.t, da_first) and torch.equal(db.t, db_first)
    for (p, q, i, t, off_t), (_, _, _, u, off_u) in zip(ahead, back):
        xs, ds = x[p:q].double(), dy[p:q].double()
        check(da.t[i], u.t() @ xs, off_u.t() @ xs.abs() + (rows + 8) * U * (u.abs().t() @ xs.abs()), "da")
        check(db.t[i], ds.t() @ t, ds.abs().t() @ off_t + (rows + 8) * U * (ds.abs().t() @ t.abs()), "db")
    assert dc.workspace_status(ws.t) == dc.OK

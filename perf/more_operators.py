"""Products of rows that belong to groups, and low-rank adapters beside a shared 1x1 layer: each one pass through the library's public
entry points, beside their plain forms.

  group     y = act(x W_g^T + b_g) of rows sorted by the group they belong to, group g having weights of its own (dc_group_forward)
  group_train    its gradients for dy: dx = dy W_g, dW_g = dy^T x, db_g = the sum of dy over the group's rows (dc_group_backward)
  adapter   y = act(x W^T + bias + residual + scale_a (x A_a^T) B_a^T): weights that all rows share, and a low-rank adapter a for each run of
            rows, that of the request which the rows come from (dc_adapter_forward); without W beside a projection made elsewhere
  adapter_train  that forward pass and its gradients for dy: dx, and dA_a, dB_a of every adapter (dc_adapter_backward)

Groups and requests are runs of rows between offsets that the GPU holds; a group may be empty, a request may have no adapter (-1) or one that
others have too, and rows behind the last run belong to none.

Shapes are those of 1x1 layers and of the classifier of the network in paper_2301_12187_b200/inputs.py, and generic ones up to 16384 rows and
4096 channels.
"""
import math

import torch

own = False                                      # whether run() makes the library's calls; set from outside

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BYTES_MAX, FLOPS_MAX, FLOPS_MAX_F32 = 7.0e8, 5.4e11, 4.0e10     # bounds on one drawn case: below the largest listed ones


# --------------------------------------------------------------------------- the cases


def listed():
    return [
        # Four tokens and eight experts: few weights are touched, latency.
        dict(name="group_token", kind="group", rows=4, groups=8, c_in=1024, c_out=1024, tail=0, dtype="bf16", bias=False, act=0),
        # A step of decoding: 256 rows over 64 experts, a few rows each; bound by reading the experts' weights.
        dict(name="group_decode", kind="group", rows=256, groups=64, c_in=2048, c_out=2048, tail=0, dtype="bf16", bias=False, act=0),
        # A long batch over 16 experts: bound by the tensor core.
        dict(name="group_prefill", kind="group", rows=16384, groups=16, c_in=4096, c_out=4096, tail=0, dtype="bf16", bias=True, act=0),
        # Odd rows and channels in fp32, ReLU6, some rows behind the last group.
        dict(name="group_ragged", kind="group", rows=3001, groups=7, c_in=500, c_out=1003, tail=13, dtype="f32", bias=True, act=1),
        # The gradients of a batch over 8 experts.
        dict(name="group_train", kind="group_train", rows=8192, groups=8, c_in=2048, c_out=4096, tail=0, dtype="bf16", bias=True),
        # The same in fp32 of the network's head, 320 -> 1280, one for each of 5 tasks: 1501 pixels.
        dict(name="group_train_head", kind="group_train", rows=1501, groups=5, c_in=320, c_out=1280, tail=5, dtype="f32", bias=True),
        # Four requests at one token each, each with an adapter of its own: latency.
        dict(name="adapter_token", kind="adapter", rows=4, requests=4, adapters=8, rank=16, c_in=4096, c_out=4096, dtype="bf16", shared=True,
             bias=False, residual=False, act=0),
        # A step of decoding for 128 requests and 96 adapters; the adapters weigh more than the shared weights.
        dict(name="adapter_decode", kind="adapter", rows=128, requests=128, adapters=96, rank=32, c_in=4096, c_out=4096, dtype="bf16", shared=True,
             bias=True, residual=False, act=0),
        # Requests that are read in beside others that decode: runs of one row and runs of hundreds.
        dict(name="adapter_mixed", kind="adapter", rows=2080, requests=40, adapters=24, rank=16, c_in=2048, c_out=2048, dtype="bf16", shared=True,
             bias=True, residual=True, act=0),
        # Six long requests: bound by the tensor core.
        dict(name="adapter_prefill", kind="adapter", rows=8192, requests=6, adapters=8, rank=64, c_in=4096, c_out=4096, dtype="bf16", shared=True,
             bias=False, residual=False, act=0),
        # The adapters' part alone, added to what a projection with 4-bit weights gave.
        dict(name="adapter_beside", kind="adapter", rows=4096, requests=9, adapters=4, rank=8, c_in=4096, c_out=1024, dtype="bf16", shared=False,
             bias=False, residual=True, act=0),
        # A step of training two adapters over frozen weights, rows of eight sequences.
        dict(name="adapter_train", kind="adapter_train", rows=8192, requests=8, adapters=2, rank=16, c_in=4096, c_out=4096, dtype="bf16", shared=True,
             bias=False, residual=False, act=0),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    """Mostly multiples of 8, as layers have them; one in five is any number."""
    v = _log_int(rng, lo, hi)
    return v if rng.random() < 0.2 else min(hi, max(8, v // 8 * 8))


def draw(rng):
    kind = rng.choice(["group", "group", "group_train", "adapter", "adapter", "adapter", "adapter_train"])
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    c_in, c_out = _width(rng, 64, 4096), _width(rng, 64, 4096)
    rows = _log_int(rng, 1, 256) if rng.random() < 0.4 else _log_int(rng, 256, 16384)
    if kind in ("group", "group_train"):
        case = dict(kind=kind, rows=rows, groups=_log_int(rng, 1, 64), c_in=c_in, c_out=c_out, tail=rng.choice([0, 0, 0, rng.randint(1, 40)]),
                    dtype=dtype, bias=rng.random() < 0.5)
        if kind == "group":
            case["act"] = int(rng.random() < 0.3)
    else:
        requests = rows if rows <= 128 and rng.random() < 0.6 else min(rows, _log_int(rng, 1, 12))
        rank = rng.choice([8, 16, 16, 32, 64, 128, rng.randint(1, 100)])
        shared = kind == "adapter_train" or rng.random() < 0.8
        case = dict(kind=kind, rows=rows, requests=requests, adapters=_log_int(rng, 1, 64), rank=rank, c_in=c_in, c_out=c_out, dtype=dtype,
                    shared=shared, bias=rng.random() < 0.5, residual=not shared or rng.random() < 0.3,
                    act=int(kind == "adapter" and rng.random() < 0.2))
    while True:
        w = work(case)
        over = max(w["bytes"] / BYTES_MAX, w["flops"] / (FLOPS_MAX if dtype == "bf16" else FLOPS_MAX_F32))
        if over <= 1.0:
            return case
        # fewer groups where their weights are what is much, else fewer rows
        if kind in ("group", "group_train") and case["groups"] > 1 and w["bytes"] > BYTES_MAX:
            case["groups"] = max(1, int(case["groups"] / max(over, 1.2)))
        elif case["rows"] > 1:
            case["rows"] = max(1, int(case["rows"] / max(over, 1.05)))
            if "requests" in case:
                case["requests"] = min(case["requests"], case["rows"])
        else:
            return case


def _elem(case):
    return 2 if case["dtype"] == "bf16" else 4


def work(case):
    e, rows, c_in, c_out = _elem(case), case["rows"], case["c_in"], case["c_out"]
    x, y = rows * c_in * e, rows * c_out * e
    if case["kind"] in ("group", "group_train"):
        # a group without rows is not read
        w = min(case["groups"], rows) * c_in * c_out * e
        bias = 4 * min(case["groups"], rows) * c_out if case["bias"] else 0
        if case["kind"] == "group":
            return {"bytes": x + w + y + bias, "flops": 2.0 * rows * c_in * c_out}
        return {"bytes": x + y + w + x + case["groups"] * c_in * c_out * e + bias, "flops": 4.0 * rows * c_in * c_out}
    used = min(case["adapters"], case["requests"])
    ab = (c_in + c_out) * case["rank"] * e
    w = c_in * c_out * e if case["shared"] else 0
    flops = (2.0 * rows * c_in * c_out if case["shared"] else 0.0) + 2.0 * rows * (c_in + c_out) * case["rank"]
    forward = x + w + used * ab + (2 if case["residual"] else 1) * y + (4 * c_out if case["bias"] else 0)
    if case["kind"] == "adapter":
        return {"bytes": forward, "flops": flops}
    # the gradients: dy, x, w and the adapters are read, dx and the adapters' gradients written
    return {"bytes": forward + y + x + w + used * ab + x + case["adapters"] * ab, "flops": 2.0 * flops + 2.0 * rows * (c_in + c_out) * case["rank"]}


# --------------------------------------------------------------------------- inputs


def _generator(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 6151 + 29)
    return g


def _sizes(case, seed):
    """How many rows each run has (host numbers): uneven, of many groups some empty; of requests each has one row at least."""
    g = torch.Generator()
    g.manual_seed(int(seed) * 7919 + 3)
    if "groups" in case:
        n, rows = case["groups"], case["rows"]
        weight = torch.exp(0.4 * torch.randn(n, generator=g, dtype=torch.float64))
        if n > 3:
            weight[int(torch.randint(n, (1,), generator=g))] = 0.0
        picks = torch.multinomial(weight, rows, replacement=True, generator=g)
        return torch.bincount(picks, minlength=n).tolist()
    n, rows = case["requests"], case["rows"]
    long_ones = n if n <= 12 else max(1, n // 8)
    weight = torch.zeros(n, dtype=torch.float64)
    weight[torch.randperm(n, generator=g)[:long_ones]] = 1.0
    weight = weight * torch.exp(0.3 * torch.randn(n, generator=g, dtype=torch.float64))
    extra = torch.bincount(torch.multinomial(weight, rows - n, replacement=True, generator=g), minlength=n) if rows > n else torch.zeros(n, dtype=torch.int64)
    return (1 + extra).tolist()


def _raw(case, seed):
    g = _generator(case, seed)
    dtype, c_in, c_out = DTYPES[case["dtype"]], case["c_in"], case["c_out"]
    sizes = _sizes(case, seed)
    rows = case["rows"] + case.get("tail", 0)
    rand = lambda *shape: torch.randn(*shape, generator=g, device="cuda")
    gain = torch.exp(0.3 * rand(c_in))
    raw = {"case": case, "used": case["rows"], "longest": max(sizes), "x": (rand(rows, c_in) * gain).to(dtype)}
    raw["offsets"] = torch.tensor([0] + torch.tensor(sizes).cumsum(0).tolist(), dtype=torch.int32, device="cuda")
    if "groups" in case:
        raw["w"] = torch.empty(case["groups"], c_out, c_in, dtype=dtype, device="cuda")
        raw["w"].normal_(0.0, 1.0 / math.sqrt(c_in), generator=g)
        raw["bias"] = rand(case["groups"], c_out) * 0.1 if case["bias"] else None
        raw["residual"] = None
    else:
        n, r = case["adapters"], case["rank"]
        raw["w"] = (rand(c_out, c_in) / math.sqrt(c_in)).to(dtype) if case["shared"] else None
        raw["bias"] = rand(c_out) * 0.1 if case["bias"] else None
        raw["residual"] = rand(rows, c_out).to(dtype) if case["residual"] else None
        raw["a"] = (rand(n, r, c_in) / math.sqrt(c_in)).to(dtype)
        raw["b"] = (rand(n, c_out, r) / math.sqrt(r)).to(dtype)
        raw["scale"] = 0.25 + 0.5 * torch.rand(n, generator=g, device="cuda")
        which = torch.randint(n, (case["requests"],), generator=g, device="cuda", dtype=torch.int32)
        if case["requests"] > 4 and case["kind"] == "adapter":
            which[1::5] = -1                     # requests without an adapter
        raw["which"] = which
    if case["kind"].endswith("train"):
        raw["dy"] = rand(rows, c_out).to(dtype)
    return raw


def prepare(case, seed):
    s = _raw(case, seed)
    s["y"] = torch.zeros(s["x"].shape[0], case["c_out"], dtype=s["x"].dtype, device="cuda")
    if case["kind"].endswith("train"):
        s["dx"] = torch.zeros_like(s["x"])
        if "groups" in case:
            s["dw"] = torch.empty_like(s["w"])
            s["db"] = torch.empty_like(s["bias"]) if s["bias"] is not None else None
        else:
            s["da"], s["db"] = torch.empty_like(s["a"]), torch.empty_like(s["b"])
    if own:
        _own_handles(s)
    return s


# --------------------------------------------------------------------------- the plain forms


def _blocks(t, place, runs, longest):
    """Rows as [runs, longest, columns], zeros behind the end of a run."""
    blocks = t.new_zeros(runs * longest, t.shape[1])
    blocks[place] = t
    return blocks.view(runs, longest, t.shape[1])


def _places(s):
    """Of every row that belongs to a run: its place in _blocks."""
    row = torch.arange(s["used"], device="cuda")
    run = torch.searchsorted(s["offsets"][1:].long(), row, right=True)
    return run * s["longest"] + row - s["offsets"].long()[run]


def _act(y, act):
    return y.clamp(0.0, 6.0) if act else y


def _rows(blocks, place, like):
    """Rows out of _blocks, zeros for those that belong to no run."""
    out = blocks.new_zeros(like.shape[0], blocks.shape[2])
    out[:place.shape[0]] = blocks.reshape(-1, blocks.shape[2])[place]
    return out


def _plain_group(s):
    case, used = s["case"], s["used"]
    place, runs = _places(s), case["groups"]
    x = _blocks(s["x"][:used].float(), place, runs, s["longest"])
    y = torch.bmm(x, s["w"].float().transpose(1, 2))
    if s["bias"] is not None:
        y = y + s["bias"][:, None]
    return _rows(_act(y, case["act"]), place, s["x"]).to(s["x"].dtype)


def _plain_group_train(s):
    dtype, used = s["x"].dtype, s["used"]
    place, runs = _places(s), s["case"]["groups"]
    x = _blocks(s["x"][:used].float(), place, runs, s["longest"])
    dy = _blocks(s["dy"][:used].float(), place, runs, s["longest"])
    out = {"dx": _rows(torch.bmm(dy, s["w"].float()), place, s["x"]).to(dtype), "dw": torch.bmm(dy.transpose(1, 2), x).to(dtype)}
    if s["bias"] is not None:
        out["db"] = dy.sum(1)
    return out


def _adapters_of(s):
    """The adapter matrices and scales of every request; scale 0 where it has none."""
    which = s["which"].long().clamp(min=0)
    scale = s["scale"][which] * (s["which"] >= 0)
    return which, s["a"][which].float(), s["b"][which].float(), scale[:, None, None]


def _plain_adapter(s):
    case, x = s["case"], s["x"].float()
    place, runs = _places(s), case["requests"]
    _, a, b, scale = _adapters_of(s)
    t = torch.bmm(_blocks(x, place, runs, s["longest"]), a.transpose(1, 2)) * scale
    y = _rows(torch.bmm(t, b.transpose(1, 2)), place, x)
    if s["w"] is not None:
        y = y + torch.matmul(x, s["w"].float().t())
    if s["bias"] is not None:
        y = y + s["bias"]
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return _act(y, case["act"]).to(s["x"].dtype)


def _plain_adapter_train(s):
    case, dtype = s["case"], s["x"].dtype
    out = {"y": _plain_adapter(s)}
    place, runs = _places(s), case["requests"]
    which, a, b, scale = _adapters_of(s)
    x, dy = _blocks(s["x"].float(), place, runs, s["longest"]), _blocks(s["dy"].float(), place, runs, s["longest"])
    t = torch.bmm(x, a.transpose(1, 2)) * scale
    u = torch.bmm(dy, b) * scale
    out["dx"] = (_rows(torch.bmm(u, a), place, s["x"]) + torch.matmul(s["dy"].float(), s["w"].float())).to(dtype)
    # requests with the same adapter are added up
    share = (which == torch.arange(case["adapters"], device="cuda")[:, None]).float()
    out["da"] = torch.matmul(share, torch.bmm(u.transpose(1, 2), x).reshape(runs, -1)).view(s["a"].shape).to(dtype)
    out["db"] = torch.matmul(share, torch.bmm(dy.transpose(1, 2), t).reshape(runs, -1)).view(s["b"].shape).to(dtype)
    return out


PLAIN = {"group": _plain_group, "group_train": _plain_group_train, "adapter": _plain_adapter, "adapter_train": _plain_adapter_train}


# --------------------------------------------------------------------------- the library's calls


def _own_handles(s):
    """What a program keeps: a workspace, and for adapters their descriptor and the buffer that the backward pass reads."""
    from paper_2301_12187_b200 import dc
    case, rows = s["case"], s["x"].shape[0]
    code = dc.dtype_code(s["x"].dtype)
    if "groups" in case:
        size = dc.group_workspace_bytes(rows, case["groups"], case["c_in"], case["c_out"], code)
    else:
        s["adapters"] = dc.Adapters(s["a"], s["b"], s["scale"])
        s["saved"] = s["adapters"].saved(rows)
        size = dc.adapter_workspace_bytes(rows, case["c_in"], case["c_out"], s["adapters"], code)
    s["ws"] = torch.zeros(size, dtype=torch.uint8, device="cuda")


def _own(s):
    from paper_2301_12187_b200 import dc
    kind, case = s["case"]["kind"], s["case"]
    if kind == "group":
        dc.group_forward(s["x"], s["offsets"], s["w"], s["bias"], case["act"], s["y"], s["ws"])
        return s["y"]
    if kind == "group_train":
        dc.group_backward(s["dy"], s["x"], s["offsets"], s["w"], s["dx"], s["dw"], s["db"], s["ws"])
        out = {"dx": s["dx"], "dw": s["dw"]}
        if s["db"] is not None:
            out["db"] = s["db"]
        return out
    dc.adapter_forward(s["x"], s["w"], s["adapters"], s["offsets"], s["which"], s["bias"], case["act"], s["residual"], s["saved"], s["y"], s["ws"])
    if kind == "adapter":
        return s["y"]
    dc.adapter_backward(s["dy"], s["x"], s["w"], s["adapters"], s["offsets"], s["which"], s["saved"], s["dx"], s["da"], s["db"], s["ws"])
    return {"y": s["y"], "dx": s["dx"], "da": s["da"], "db": s["db"]}


def run(state):
    return _own(state) if own else PLAIN[state["case"]["kind"]](state)


# --------------------------------------------------------------------------- from the definition, in 64 bits


def exact(case, seed):
    """Run by run: each of them on its own rows, in double precision."""
    s = _raw(case, seed)
    x, bounds = s["x"].double(), s["offsets"].tolist()
    y = torch.zeros(x.shape[0], case["c_out"], dtype=torch.float64, device="cuda")
    runs = list(zip(bounds[:-1], bounds[1:]))
    train = case["kind"].endswith("train")
    dy = s["dy"].double() if train else None
    dx = torch.zeros_like(x)
    if "groups" in case:
        dw = torch.zeros(s["w"].shape, dtype=torch.float64, device="cuda")
        db = torch.zeros(case["groups"], case["c_out"], dtype=torch.float64, device="cuda")
        for g, (lo, hi) in enumerate(runs):
            w = s["w"][g].double()
            if train:
                dx[lo:hi] = dy[lo:hi] @ w
                dw[g] = dy[lo:hi].t() @ x[lo:hi]
                db[g] = dy[lo:hi].sum(0)
            else:
                y[lo:hi] = x[lo:hi] @ w.t() + (s["bias"][g].double() if case["bias"] else 0.0)
                if case["act"]:
                    y[lo:hi] = y[lo:hi].clamp(0, 6)
        if not train:
            return y
        return {"dx": dx, "dw": dw, "db": db} if case["bias"] else {"dx": dx, "dw": dw}
    if case["shared"]:
        w = s["w"].double()
        y = x @ w.t()
        if train:
            dx = dy @ w
    da, db = torch.zeros(s["a"].shape, dtype=torch.float64, device="cuda"), torch.zeros(s["b"].shape, dtype=torch.float64, device="cuda")
    for (lo, hi), k in zip(runs, s["which"].tolist()):
        if k < 0:
            continue
        a, b, scale = s["a"][k].double(), s["b"][k].double(), float(s["scale"][k])
        y[lo:hi] += scale * ((x[lo:hi] @ a.t()) @ b.t())
        if train:
            dx[lo:hi] += scale * ((dy[lo:hi] @ b) @ a)
            da[k] += scale * ((dy[lo:hi] @ b).t() @ x[lo:hi])
            db[k] += scale * (dy[lo:hi].t() @ (x[lo:hi] @ a.t()))
    if case["bias"]:
        y = y + s["bias"].double()
    if case["residual"]:
        y = y + s["residual"].double()
    if case["act"]:
        y = y.clamp(0, 6)
    return {"y": y, "dx": dx, "da": da, "db": db} if train else y

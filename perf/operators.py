"""Performance cases of the network operators: group normalisation of
channels-last maps and a projection that many cameras or requests share, each
with its own low-rank adapter, forward and backward.

Kinds of case ("kind"):
  norm       nsc_group_norm: one map per image, statistics per image and group
  norm_grad  nsc_group_norm_backward
  lora       nsc_adapter_project: rows of many adapters beside one projection
  lora_grad  nsc_adapter_backward

Map sizes and channel counts are those of the networks in synth/workloads.py
(50 x 50, 25 x 25 and 12 x 12 maps of 32 and 64 channels), then wider and odd
ones; projections are those networks' dense layers (a flattened map onto 32 to
128 units) and square ones of a few thousand.  Without the library's operators
(`own` false) `run` computes the same with elementary torch operations.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-5


def _norm(name, n, h, w, c, groups, dtype, act, kind="norm", live=None, pad=0):
    """live: images the device-side count leaves of the n there is room for;
    pad: elements between one image's end and the next one's start."""
    return dict(name=name, kind=kind, n=n, h=h, w=w, c=c, groups=groups, dtype=dtype, act=act,
                live=n if live is None else live, pad=pad)


def _lora(name, n, k, d, rank, adapters, dtype, order, kind="lora", live=None, pad=0):
    """order: how the rows' adapters come (see _ids)."""
    return dict(name=name, kind=kind, n=n, k=k, d=d, rank=rank, adapters=adapters, dtype=dtype,
                order=order, live=n if live is None else live, pad=pad)


def listed():
    return [
        # one survivor's pooled map between two layers of a live stream: latency
        _norm("norm-one-frame", 1, 25, 25, 32, 8, "f32", "relu"),
        # the survivors of a busy chunk, first map of the 64-channel networks, a
        # ragged number of them in a larger buffer
        _norm("norm-survivors", 1200, 50, 50, 64, 8, "bf16", "relu", live=1031),
        # a few wide maps at a finer grid, smooth activation
        _norm("norm-wide-maps", 4, 112, 112, 320, 32, "f16", "silu"),
        # channels that fill no 16-byte vectors, images that are not adjacent
        _norm("norm-odd-channels", 300, 37, 41, 45, 5, "bf16", "none", pad=3),
        # one training step's batch through the same layer
        _norm("norm-grad-batch", 512, 50, 50, 64, 8, "bf16", "relu", kind="norm_grad"),
        # a small fp32 batch of pooled maps
        _norm("norm-grad-fp32", 48, 25, 25, 32, 8, "f32", "silu", kind="norm_grad"),
        # one survivor of one camera through the dense layer: latency
        _lora("adapter-one-row", 1, 4608, 128, 8, 24, "bf16", "sorted"),
        # the survivors of a second of 100 cameras, camera by camera
        _lora("adapter-cameras", 500, 4608, 128, 8, 100, "bf16", "sorted"),
        # one row of each of 64 requests in any order, some without an adapter
        _lora("adapter-requests", 64, 4096, 4096, 16, 32, "f16", "mixed"),
        # many rows of a few dozen requests, request by request, ragged lengths
        _lora("adapter-long", 4096, 4096, 4096, 16, 24, "bf16", "runs"),
        # fitting cameras' adapters of the 4-layer network's dense layer, fp32
        _lora("adapter-grad", 1501, 9216, 128, 16, 24, "f32", "runs", kind="lora_grad"),
        # the same for requests in any order over a wide square projection
        _lora("adapter-grad-mixed", 2000, 2048, 2048, 16, 12, "bf16", "mixed", kind="lora_grad",
              pad=8),
    ]


def draw(rng):
    """One more case of the same kinds: sizes log-uniform, odd ones among them."""
    def size(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["norm", "norm", "norm_grad", "lora", "lora", "lora_grad"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if kind.startswith("norm"):
        c = rng.choice([16, 32, 64, 64, 8 * size(1, 64), size(3, 130)])
        groups = rng.choice([g for g in range(1, c + 1) if c % g == 0])
        h = rng.choice([12, 25, 50, size(3, 112)])
        w = h if rng.random() < 0.5 else size(3, 112)
        # a row of buffers costs no more than the largest listed one
        most = (1.6e8 if kind == "norm" else 8e7) * (0.5 if dtype == "f32" else 1) / (h * w * c)
        n = size(1, max(1, min(2048, int(most))))
        case = _norm("", n, h, w, c, groups, dtype, rng.choice(["relu", "relu", "silu", "none"]),
                     kind, live=n if rng.random() < 0.7 else rng.randint(1, n),
                     pad=rng.choice([0, 0, 8, 8, 5]))
        del case["name"]
        return case
    k = rng.choice([2304, 4608, 9216, 8 * size(8, 1024), size(64, 4096)])
    d = rng.choice([32, 64, 128, 128, 8 * size(4, 512), size(16, 512)])
    rank = rng.choice([4, 8, 16, 32, size(1, 64)])
    most = (1.2e11 if kind == "lora" else 4e10) * (0.1 if dtype == "f32" else 1) / (2 * k * d)
    n = size(1, max(1, min(4096, int(most))))
    case = _lora("", n, k, d, rank, size(1, 128), dtype, rng.choice(["sorted", "mixed", "runs"]),
                 kind, live=n if rng.random() < 0.7 else rng.randint(1, n),
                 pad=rng.choice([0, 0, 8, 3]))
    del case["name"]
    return case


# ------------------------------------------------------------------ inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _rows(n, width, pad, dtype, fill=None):
    """n rows `width` wide, `pad` elements apart, zeros or the given values."""
    buf = torch.zeros((n, width + pad), dtype=TYPES[dtype], device=DEV)
    if fill is not None:
        buf[:, :width] = fill
    return buf


def _maps(case, g):
    """Pre-activation maps: a mean and spread per channel, a brightness per image."""
    n, hw, c = case["n"], case["h"] * case["w"], case["c"]
    mean = torch.randn(c, device=DEV, generator=g) * 0.7
    spread = torch.rand(c, device=DEV, generator=g) + 0.3
    gain = torch.rand((n, 1, 1), device=DEV, generator=g) + 0.5
    x = torch.randn((n, hw, c), device=DEV, generator=g)
    return x.mul_(spread).add_(mean).mul_(gain).view(n, hw * c)


def _ids(case, g):
    """The rows' adapters.  "sorted": camera by camera, in adapter order;
    "runs": request by request, ragged, in any order; "mixed": a row at a time
    in any order.  About a tenth of the runs and mixed rows have none (-1)."""
    n, m, order = case["n"], case["adapters"], case["order"]
    if order == "mixed":
        ids = torch.randint(0, m, (n,), device=DEV, generator=g)
        none = torch.rand(n, device=DEV, generator=g) < 0.1
    else:
        runs = max(1, min(n, m))
        cuts = torch.randint(0, n + 1, (runs - 1,), device=DEV, generator=g).sort().values
        run = torch.searchsorted(cuts, torch.arange(n, device=DEV), right=True)
        if order == "sorted":
            return run.int()
        ids = torch.randperm(m, device=DEV, generator=g)[run]
        none = (torch.rand(runs, device=DEV, generator=g) < 0.1)[run]
    return torch.where(none, -1, ids).int()


def prepare(case, seed):
    g = _gen(seed)
    t, n = case["dtype"], case["n"]
    s = dict(case=case, count=torch.tensor([case["live"]], dtype=torch.int32, device=DEV))
    if case["kind"].startswith("norm"):
        c, width = case["c"], case["h"] * case["w"] * case["c"]
        s["x"] = _rows(n, width, case["pad"], t, _maps(case, g))
        s["gamma"] = 1 + 0.2 * torch.randn(c, device=DEV, generator=g)
        s["beta"] = 0.3 * torch.randn(c, device=DEV, generator=g)
        if case["kind"] == "norm":
            s["y"] = _rows(n, width, case["pad"], t)
            s["stats"] = torch.zeros((n, case["groups"], 2), device=DEV)
        else:  # the statistics that the forward pass left
            s["dy"] = _rows(n, width, case["pad"], t,
                            torch.randn((n, width), device=DEV, generator=g))
            mean, rstd = _moments(_grouped(s["x"], case))
            s["stats"] = torch.stack([mean, rstd], -1).view(n, case["groups"], 2)
            s["dx"] = _rows(n, width, case["pad"], t)
            s["dgamma"], s["dbeta"] = (torch.zeros(c, device=DEV) for _ in range(2))
    else:
        k, d, r, m = case["k"], case["d"], case["rank"], case["adapters"]

        def normal(*shape, std):
            return (torch.randn(shape, device=DEV, generator=g) * std).to(TYPES[t])

        s["x"] = _rows(n, k, case["pad"], t,
                       torch.randn((n, k), device=DEV, generator=g).clamp_(min=-0.5))
        s["w"] = normal(d, k, std=1 / math.sqrt(k))
        s["bias"] = 0.1 * torch.randn(d, device=DEV, generator=g)
        s["a"] = normal(m, r, k, std=1 / math.sqrt(k))
        s["b"] = normal(m, d, r, std=0.5 / math.sqrt(r))
        s["scale"] = 0.5 + torch.rand(m, device=DEV, generator=g)
        s["ids"] = _ids(case, g)
        if case["kind"] == "lora":
            s["y"] = _rows(n, d, case["pad"], t)
        else:
            s["dy"] = _rows(n, d, case["pad"], t, torch.randn((n, d), device=DEV, generator=g))
            s["dx"] = _rows(n, k, case["pad"], t)
            s["da"] = torch.zeros((m, r, k), device=DEV)
            s["db"] = torch.zeros((m, d, r), device=DEV)
    if own:
        _plan(s)
    return s


# ------------------------------------------------- the library's operators

def _plan(s):
    """The description and workspace that a program keeps beside its buffers."""
    import paper_1703_02529_amd as nsc
    case = s["case"]
    dtype = {"f32": nsc.NSC_T_F32, "bf16": nsc.NSC_T_BF16, "f16": nsc.NSC_T_F16}[case["dtype"]]
    grad = case["kind"].endswith("_grad")
    if case["kind"].startswith("norm"):
        act = {"none": nsc.NSC_ACT_NONE, "relu": nsc.NSC_ACT_RELU, "silu": nsc.NSC_ACT_SILU}
        stride = s["x"].shape[1]
        s["desc"] = nsc.make_norm_desc(case["h"], case["w"], case["c"], case["groups"],
                                       act=act[case["act"]], dtype=dtype, eps=EPS,
                                       x_stride=stride, y_stride=stride)
        size = nsc.nsc_group_norm_workspace_bytes(s["desc"], case["n"], backward=grad)
    else:
        s["desc"] = nsc.make_adapter_desc(case["k"], case["d"], case["rank"], case["adapters"],
                                          dtype=dtype, x_stride=s["x"].shape[1],
                                          y_stride=s["dy" if grad else "y"].shape[1])
        size = nsc.nsc_adapter_workspace_bytes(s["desc"], case["n"], backward=grad)
    s["ws"] = torch.empty(max(size, 256), dtype=torch.uint8, device=DEV)
    s["nsc"] = nsc


def _run_own(s):
    nsc, kind, n = s["nsc"], s["case"]["kind"], s["case"]["n"]
    if kind == "norm":
        nsc.nsc_group_norm(s["desc"], s["x"], s["gamma"], s["beta"], s["y"], s["ws"], n,
                           stats=s["stats"], count=s["count"])
        return dict(y=s["y"], stats=s["stats"])
    if kind == "norm_grad":
        nsc.nsc_group_norm_backward(s["desc"], s["x"], s["dy"], s["gamma"], s["beta"], s["stats"],
                                    s["dx"], s["dgamma"], s["dbeta"], s["ws"], n,
                                    count=s["count"])
        return dict(dx=s["dx"], dgamma=s["dgamma"], dbeta=s["dbeta"])
    if kind == "lora":
        nsc.nsc_adapter_project(s["desc"], s["x"], s["w"], s["bias"], s["a"], s["b"], s["scale"],
                                s["ids"], s["y"], s["ws"], n, count=s["count"])
        return dict(y=s["y"])
    nsc.nsc_adapter_backward(s["desc"], s["x"], s["dy"], s["w"], s["a"], s["b"], s["scale"],
                             s["ids"], s["dx"], s["da"], s["db"], s["ws"], n, count=s["count"])
    return dict(dx=s["dx"], da=s["da"], db=s["db"])


# ------------------------------------------------------- elementary torch

def _grouped(buf, case):
    """fp32 maps [image, pixel, group, channel of the group]."""
    n, g = case["n"], case["groups"]
    x = buf[:, :case["h"] * case["w"] * case["c"]].float()
    return x.reshape(n, case["h"] * case["w"], g, case["c"] // g)


def _moments(x):
    mean = x.mean((1, 3), keepdim=True)
    var = (x - mean).square().mean((1, 3), keepdim=True)
    return mean, 1 / torch.sqrt(var + EPS)


def _live(s):
    """Whether each row lies before the device-side count, [n, 1]."""
    return (torch.arange(s["case"]["n"], device=DEV) < s["count"])[:, None]


def _store(buf, values, live):
    """Live rows of the values, rounded once; rows behind the last keep theirs."""
    width = values.shape[1]
    buf[:, :width] = torch.where(live, values.to(buf.dtype), buf[:, :width])
    return buf


def _run_norm(s):
    case = s["case"]
    n, c = case["n"], case["c"]
    x, live = _grouped(s["x"], case), _live(s)
    mean, rstd = _moments(x)
    y = ((x - mean) * rstd).view(n, -1, c) * s["gamma"] + s["beta"]
    if case["act"] == "relu":
        y = y * (y > 0)
    elif case["act"] == "silu":
        y = y / (1 + torch.exp(-y))
    stats = torch.stack([mean, rstd], -1).view(n, -1)
    _store(s["stats"].view(n, -1), stats, live)
    return dict(y=_store(s["y"], y.view(n, -1), live), stats=s["stats"])


def _run_norm_grad(s):
    case = s["case"]
    n, c, g = case["n"], case["c"], case["groups"]
    x, live = _grouped(s["x"], case), _live(s)
    mean, rstd = (s["stats"][:, :, i].reshape(n, 1, g, 1) for i in (0, 1))
    xh = (x - mean) * rstd
    dz = torch.where(live[:, :, None], s["dy"][:, :xh[0].numel()].float().view(n, -1, c), 0.0)
    gamma, beta = s["gamma"], s["beta"]
    if case["act"] == "relu":  # the sign of values next to zero: 64 bits
        z = ((x.double() - mean) * rstd.double()).view(n, -1, c) * gamma.double() + beta
        dz = dz * (z > 0)
    elif case["act"] == "silu":
        z = xh.view(n, -1, c) * gamma + beta
        p = 1 / (1 + torch.exp(-z))
        dz = dz * p * (1 + z * (1 - p))
    s["dbeta"].copy_(dz.sum((0, 1), dtype=torch.float64))
    s["dgamma"].copy_((dz * xh.view(n, -1, c)).sum((0, 1), dtype=torch.float64))
    gz = (dz * gamma).view_as(x)
    dx = rstd * (gz - gz.mean((1, 3), keepdim=True) - xh * (gz * xh).mean((1, 3), keepdim=True))
    return dict(dx=_store(s["dx"], dx.reshape(n, -1), live), dgamma=s["dgamma"], dbeta=s["dbeta"])


def _chosen(s):
    """Each live row's factor on each adapter's columns, [n, adapters, 1]: its
    scale at its own adapter, else zero."""
    m = s["case"]["adapters"]
    hit = (s["ids"][:, None] == torch.arange(m, device=DEV)) & _live(s)
    return (hit * s["scale"])[:, :, None]


def _products(s):
    """fp32 operands: x, W, every adapter's A rows [m r, k] and B columns [d, m r]."""
    case = s["case"]
    a = s["a"].float().view(-1, case["k"])
    b = s["b"].float().permute(1, 0, 2).reshape(case["d"], -1)
    return s["x"][:, :case["k"]].float(), s["w"].float(), a, b


def _run_lora(s):
    case = s["case"]
    x, w, a, b = _products(s)
    t = torch.matmul(x, a.t()).view(case["n"], case["adapters"], -1) * _chosen(s)
    y = torch.matmul(x, w.t()) + s["bias"] + torch.matmul(t.view(case["n"], -1), b.t())
    return dict(y=_store(s["y"], y, _live(s)))


def _run_lora_grad(s):
    case = s["case"]
    n, m, r, d = case["n"], case["adapters"], case["rank"], case["d"]
    x, w, a, b = _products(s)
    pick, live = _chosen(s), _live(s)
    # rows behind the count may hold anything: they add nothing to the sums
    x, dy = torch.where(live, x, 0.0), torch.where(live, s["dy"][:, :d].float(), 0.0)
    t = (torch.matmul(x, a.t()).view(n, m, r) * pick).view(n, -1)
    u = (torch.matmul(dy, b).view(n, m, r) * pick).view(n, -1)
    dx = torch.matmul(dy, w) + torch.matmul(u, a)
    s["da"].copy_(torch.matmul(u.t(), x).view(m, r, -1))
    s["db"].copy_(torch.matmul(dy.t(), t).view(d, m, r).permute(1, 0, 2))
    return dict(dx=_store(s["dx"], dx, live), da=s["da"], db=s["db"])


def run(state):
    if own:
        return _run_own(state)
    return globals()["_run_" + state["case"]["kind"]](state)


# -------------------------------------------------------------------- work

def _used(case):
    """Adapters that can have a row, and the rows."""
    return min(case["adapters"], case["live"]), case["live"]


def work(case):
    es = 4 if case["dtype"] == "f32" else 2
    if case["kind"].startswith("norm"):
        e = case["live"] * case["h"] * case["w"] * case["c"]
        small = 8 * case["live"] * case["groups"] + 8 * case["c"]
        if case["kind"] == "norm":
            return dict(bytes=2 * es * e + small, flops=8.0 * e)
        return dict(bytes=3 * es * e + small + 8 * case["c"], flops=16.0 * e)
    k, d, r = case["k"], case["d"], case["rank"]
    m, n = _used(case)
    # a live row reads its input and writes its output; weights are read once
    if case["kind"] == "lora":
        return dict(bytes=es * (n * (k + d) + d * k + m * r * (k + d)) + 4 * (d + n),
                    flops=2.0 * n * (k * d + r * (k + d)))
    return dict(bytes=es * (n * (2 * k + d) + d * k + m * r * (k + d)) + 4 * n +
                4 * case["adapters"] * r * (k + d),
                flops=2.0 * n * (k * d + r * (3 * k + 2 * d)))


# ------------------------------------------------------------------- exact

def exact(case, seed):
    s = prepare(case, seed)
    live, n = case["live"], case["n"]
    f64 = torch.float64
    if case["kind"].startswith("norm"):
        hw, c, g = case["h"] * case["w"], case["c"], case["groups"]
        gamma, beta = s["gamma"].to(f64), s["beta"].to(f64)
        if case["kind"] == "norm":
            y, stats = torch.zeros(s["y"].shape, dtype=f64, device=DEV), s["stats"].to(f64)
        else:
            dx = torch.zeros(s["dx"].shape, dtype=f64, device=DEV)
            dgamma, dbeta = torch.zeros(c, dtype=f64, device=DEV), torch.zeros(c, dtype=f64,
                                                                               device=DEV)
        step = max(1, int(2e7 / (hw * c)))
        for i in range(0, live, step):  # images by the batch, channels first
            j = min(live, i + step)
            x = s["x"][i:j, :hw * c].to(f64).view(j - i, hw, c).transpose(1, 2)
            x = x.reshape(j - i, g, -1)
            if case["kind"] == "norm":
                mean = x.sum(2, keepdim=True) / x.shape[2]
                rstd = (((x - mean) ** 2).sum(2, keepdim=True) / x.shape[2] + EPS) ** -0.5
            else:
                mean, rstd = s["stats"][i:j].to(f64).split(1, 2)
            xh = ((x - mean) * rstd).reshape(j - i, c, hw)
            z = gamma[:, None] * xh + beta[:, None]
            sig = torch.sigmoid(z)
            if case["kind"] == "norm":
                v = {"none": z, "relu": z.clamp(min=0), "silu": z * sig}[case["act"]]
                y[i:j, :hw * c] = v.transpose(1, 2).reshape(j - i, -1)
                stats[i:j] = torch.cat([mean, rstd], 2)
                continue
            slope = {"none": torch.ones_like(z), "relu": (z > 0).to(f64),
                     "silu": sig + z * sig * (1 - sig)}[case["act"]]
            dz = s["dy"][i:j, :hw * c].to(f64).view(j - i, hw, c).transpose(1, 2) * slope
            dbeta += dz.sum((0, 2))
            dgamma += (dz * xh).sum((0, 2))
            q, p = (gamma[:, None] * dz).reshape(x.shape), xh.reshape(x.shape)
            v = q - q.mean(2, keepdim=True) - p * (q * p).mean(2, keepdim=True)
            v = (v * rstd).reshape(j - i, c, hw).transpose(1, 2).reshape(j - i, -1)
            dx[i:j, :hw * c] = v
        out = dict(y=y, stats=stats) if case["kind"] == "norm" else dict(dx=dx, dgamma=dgamma,
                                                                         dbeta=dbeta)
        return out
    x, w = s["x"][:, :case["k"]].to(f64), s["w"].to(f64)
    ids = s["ids"].clone()
    ids[live:] = -2  # behind the count: not touched
    rows = [torch.nonzero(ids == a).view(-1) for a in range(case["adapters"])]
    if case["kind"] == "lora":
        y = torch.zeros(s["y"].shape, dtype=f64, device=DEV)
        y[:live, :case["d"]] = x[:live] @ w.t() + s["bias"].to(f64)
        for a, at in enumerate(rows):
            t = x[at] @ s["a"][a].to(f64).t() * s["scale"][a].to(f64)
            y[at, :case["d"]] += t @ s["b"][a].to(f64).t()
        return dict(y=y)
    dy = s["dy"][:, :case["d"]].to(f64)
    dx = torch.zeros(s["dx"].shape, dtype=f64, device=DEV)
    da, db = s["da"].to(f64), s["db"].to(f64)
    dx[:live, :case["k"]] = dy[:live] @ w
    for a, at in enumerate(rows):
        fa, fb, q = s["a"][a].to(f64), s["b"][a].to(f64), s["scale"][a].to(f64)
        u = dy[at] @ fb * q
        dx[at, :case["k"]] += u @ fa
        da[a] = u.t() @ x[at]
        db[a] = dy[at].t() @ (x[at] @ fa.t() * q)
    return dict(dx=dx, da=da, db=db)

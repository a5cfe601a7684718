"""GPU tests of nsc_adapter_project and nsc_adapter_backward against fp64."""
import math

import pytest
import torch

import paper_1703_02529_amd as nsc

pytestmark = pytest.mark.gpu

TYPES = {"f32": (nsc.NSC_T_F32, torch.float32), "bf16": (nsc.NSC_T_BF16, torch.bfloat16),
         "f16": (nsc.NSC_T_F16, torch.float16)}
U = 2.0 ** -24   # half a step of fp32
SENTINEL = 7.0


def make_ids(order, n, m, g):
    if order == "mixed":
        ids = torch.randint(0, m, (n,), generator=g)
        return torch.where(torch.rand(n, generator=g) < 0.2, -1, ids)
    if order == "none":
        return torch.full((n,), -1)
    if order == "wild":  # anything a caller may leave there
        return torch.tensor([-1, m, -2 ** 31, 2 ** 31 - 1, 0, m - 1])[torch.randint(0, 6, (n,),
                                                                                    generator=g)]
    if order == "last":
        return torch.full((n,), m - 1)
    cuts = torch.randint(0, n + 1, (m - 1,), generator=g).sort().values
    run = torch.searchsorted(cuts, torch.arange(n), right=True)
    return run if order == "sorted" else torch.randperm(m, generator=g)[run]


class Rows:
    def __init__(self, n, k, d, rank, m, dtype="bf16", order="mixed", pad=0, shift=0, live=None,
                 bias=True, seed=0):
        self.n, self.k, self.d, self.rank, self.m = n, k, d, rank, m
        code, self.t = TYPES[dtype]
        self.live = n if live is None else min(max(live, 0), n)
        self.pad, self.shift = pad, shift
        g = torch.Generator().manual_seed(seed)
        r = lambda *s: torch.randn(s, generator=g)
        self.x = self._rows(r(n, k))
        self.dy = self._rows(r(n, d))
        self.w = self._flat(r(d, k) / math.sqrt(k))
        self.a = self._flat(r(m, rank, k) / math.sqrt(k))
        self.b = self._flat(r(m, d, rank) / math.sqrt(rank))
        self.bias = r(d).cuda() if bias else None
        self.scale = (0.5 + torch.rand(m, generator=g)).cuda()
        self.ids = make_ids(order, n, m, g).int().cuda()
        self.y, self.dx = self._rows(n, d), self._rows(n, k)
        self.da = torch.full((m, rank, k), SENTINEL, device="cuda")
        self.db = torch.full((m, d, rank), SENTINEL, device="cuda")
        self.count = None if live is None else torch.tensor([live], dtype=torch.int32).cuda()
        self.desc = nsc.make_adapter_desc(k, d, rank, m, dtype=code, x_stride=k + pad,
                                          y_stride=d + pad)
        size = max(nsc.nsc_adapter_workspace_bytes(self.desc, n, backward=b) for b in (0, 1))
        self.ws = torch.empty(max(256, size), dtype=torch.uint8, device="cuda")

    def _rows(self, v, width=None):
        n, width = v.shape if width is None else (v, width)
        buf = torch.full((self.shift + n * (width + self.pad),), SENTINEL, dtype=self.t,
                         device="cuda")[self.shift:]
        if isinstance(v, torch.Tensor):
            buf.view(n, width + self.pad)[:, :width] = v.cuda().to(self.t)
        return buf

    def _flat(self, v):
        buf = torch.empty(self.shift + v.numel(), dtype=self.t, device="cuda")[self.shift:]
        buf.copy_(v.reshape(-1))
        return buf

    def view(self, buf, width):
        return buf.view(self.n, width + self.pad)[:, :width]

    def forward(self, stream=None):
        nsc.nsc_adapter_project(self.desc, self.x, self.w, self.bias, self.a, self.b, self.scale,
                                self.ids, self.y, self.ws, self.n, count=self.count, stream=stream)

    def backward(self, stream=None, dx=True):
        nsc.nsc_adapter_backward(self.desc, self.x, self.dy, self.w, self.a, self.b, self.scale,
                                 self.ids, self.dx if dx else None, self.da, self.db, self.ws,
                                 self.n, count=self.count, stream=stream)

    def f64(self):
        w = self.w.double().cpu().view(self.d, self.k)
        a = self.a.double().cpu().view(self.m, self.rank, self.k)
        b = self.b.double().cpu().view(self.m, self.d, self.rank)
        x = self.view(self.x, self.k)[:self.live].double().cpu()
        dy = self.view(self.dy, self.d)[:self.live].double().cpu()
        return x, dy, w, a, b, self.scale.double().cpu(), self.ids[:self.live].cpu()


def chain(length):
    """fp32 roundings one after another in a sum of products over `length`, in
    any of the kernels' orders: an MFMA's own products (at most 32), its steps
    (of at least 16), and 64 for the joining of waves and parts."""
    return (32 + math.ceil(length / 16) + 64) * U


def near(got, want, tol, t):
    half = torch.finfo(t).eps / 2
    tol = (1 + half) * tol + half * want.abs() + (2.0 ** -25 if t == torch.float16 else 0)
    over = (got.double().cpu() - want).abs() - tol
    assert not (over > 0).any(), (over.max().item(), (over > 0).sum().item())


def check_forward(r):
    x, _, w, a, b, scale, ids = r.f64()
    y, mag = x @ w.t(), x.abs() @ w.abs().t()
    tol = chain(r.k) * mag
    if r.bias is not None:
        y = y + r.bias.double().cpu()
        tol = tol + U * y.abs()
    for p in range(r.m):
        at = torch.nonzero(ids == p).view(-1)
        t, tm = scale[p] * (x[at] @ a[p].t()), scale[p] * (x[at].abs() @ a[p].abs().t())
        y[at] += t @ b[p].t()
        # t's own sum and its scale, then the sum over the rank
        tol[at] += (chain(r.k) + U + chain(r.rank) + 2 * U) * (tm @ b[p].abs().t())
    tol = tol + 2 * U * y.abs()
    near(r.view(r.y, r.d)[:r.live], y, tol, r.t)


def check_backward(r, dx=True):
    x, dy, w, a, b, scale, ids = r.f64()
    gx, gtol = dy @ w, chain(r.d) * (dy.abs() @ w.abs())
    for p in range(r.m):
        at = torch.nonzero(ids == p).view(-1)
        t, tm = scale[p] * (x[at] @ a[p].t()), scale[p] * (x[at].abs() @ a[p].abs().t())
        u, um = scale[p] * (dy[at] @ b[p]), scale[p] * (dy[at].abs() @ b[p].abs())
        gx[at] += u @ a[p]
        gtol[at] += (chain(r.d) + chain(r.rank) + 4 * U) * (um @ a[p].abs())
        n = len(at)
        near(r.da[p], u.t() @ x[at], (chain(r.d) + chain(n) + 2 * U) * (um.t() @ x[at].abs()),
             torch.float32)
        near(r.db[p], dy[at].t() @ t, (chain(r.k) + chain(n) + 2 * U) * (dy[at].abs().t() @ tm),
             torch.float32)
    if dx:
        near(r.view(r.dx, r.k)[:r.live], gx, gtol + 2 * U * gx.abs(), r.t)


def untouched(r, buf, width):
    full = buf.view(r.n, width + r.pad).float().cpu()
    assert (full[r.live:] == SENTINEL).all()
    assert (full[:, width:] == SENTINEL).all()


FORMS = [  # rows, k, d, rank, adapters
    (1, 4608, 128, 8, 24), (1, 1, 1, 1, 1), (3, 7, 5, 2, 2), (16, 64, 16, 16, 4),
    (17, 100, 33, 5, 3), (64, 512, 512, 16, 32), (65, 72, 200, 17, 7), (33, 40, 24, 128, 3),
    (130, 520, 72, 33, 9), (500, 2304, 64, 8, 100), (300, 256, 640, 64, 2), (129, 1000, 130, 4, 5),
    (257, 96, 1032, 12, 40),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("order", ["sorted", "runs", "mixed"])
@pytest.mark.parametrize("form", FORMS, ids=str)
def test_forward_and_backward(form, order, dtype):
    r = Rows(*form, dtype=dtype, order=order, seed=sum(form))
    r.forward()
    check_forward(r)
    r.backward()
    check_backward(r)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("form", [(2050, 1152, 1088, 16, 6), (1100, 776, 520, 24, 70),
                                  (1030, 136, 8264, 16, 6), (1030, 8260, 140, 24, 5),
                                  (32900, 1032, 40, 8, 5)], ids=str)
def test_many_rows(form, dtype):
    r = Rows(*form, dtype=dtype, order="mixed")
    r.forward()
    check_forward(r)
    r.backward()
    check_backward(r)


@pytest.mark.parametrize("order", ["none", "wild", "last"])
def test_rows_without_adapters_and_ids_out_of_range(order):
    r = Rows(70, 136, 72, 9, 6, order=order)
    r.forward()
    check_forward(r)
    r.backward()
    check_backward(r)
    used = set(r.ids.tolist())
    for p in range(6):
        if p not in used:
            assert (r.da[p] == 0).all() and (r.db[p] == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad,shift", [(8, 0), (3, 0), (0, 1), (8, 8), (1, 5)])
@pytest.mark.parametrize("live", [None, 0, 1, 19, 40, 99, -3])
def test_strides_alignment_and_counts(dtype, pad, shift, live):
    r = Rows(40, 128, 96, 16, 4, dtype=dtype, pad=pad, shift=shift, live=live, bias=pad != 3)
    r.forward()
    check_forward(r)
    untouched(r, r.y, r.d)
    r.backward()
    check_backward(r)
    untouched(r, r.dx, r.k)


def test_the_gradient_of_the_input_is_optional():
    r = Rows(50, 64, 48, 8, 3)
    r.backward(dx=False)
    check_backward(r, dx=False)
    assert (r.dx == SENTINEL).all()


@pytest.mark.parametrize("value", [math.nan, math.inf])
@pytest.mark.parametrize("form", [(40, 128, 80, 16, 5), (700, 256, 320, 16, 5)], ids=str)
def test_not_a_number_stays_in_its_row_and_adapter(value, form):
    r = Rows(*form)
    r.ids[3] = 2
    r.forward()
    r.backward()
    y, dx, da, db = r.y.clone(), r.dx.clone(), r.da.clone(), r.db.clone()
    # a row's values: the other rows keep their results, the other adapters their gradients
    x = r.x.clone()
    r.view(r.x, r.k)[3, 5] = value
    r.forward()
    r.backward()
    rows = torch.arange(r.n, device="cuda") != 3
    keep = torch.arange(r.m, device="cuda") != 2
    assert torch.equal(r.view(r.y, r.d)[rows], r.view(y, r.d)[rows])
    assert not torch.isfinite(r.view(r.y, r.d)[3]).any()
    assert torch.equal(r.dx, dx) and torch.equal(r.da[keep], da[keep])
    assert torch.equal(r.db[keep], db[keep])
    r.x.copy_(x)
    # an adapter's values: rows of other adapters keep their results
    for t in (r.a, r.b):
        old = t.clone()
        t.view(r.m, -1)[2, 7] = value
        r.forward()
        r.backward()
        other = r.ids != 2
        assert torch.equal(r.view(r.y, r.d)[other], r.view(y, r.d)[other])
        assert torch.equal(r.view(r.dx, r.k)[other], r.view(dx, r.k)[other])
        assert torch.equal(r.da[keep], da[keep]) and torch.equal(r.db[keep], db[keep])
        t.copy_(old)


def test_rows_behind_the_count_are_not_read():
    r = Rows(40, 128, 80, 16, 5, live=21)
    r.forward()
    r.backward()
    want = [t.clone() for t in (r.y, r.dx, r.da, r.db)]
    r.view(r.x, r.k)[21:] = math.nan
    r.view(r.dy, r.d)[21:] = math.nan
    r.forward()
    r.backward()
    for t, v in zip((r.y, r.dx, r.da, r.db), want):
        assert torch.equal(t, v)


def test_backward_against_differences():
    """Gradients along directions against differences of the fp64 product (linear
    in x, and in a and b one at a time: the difference is exact)."""
    r = Rows(30, 40, 24, 6, 4, dtype="f32", order="mixed", seed=4)
    r.backward()
    x, dy, w, a, b, scale, ids = r.f64()

    def loss(x, a, b):
        y = x @ w.t()
        for p in range(4):
            at = ids == p
            y[at] += scale[p] * (x[at] @ a[p].t()) @ b[p].t()
        return (y * dy).sum()

    g = torch.Generator().manual_seed(9)
    vx, va, vb = (torch.randn(t.shape, generator=g, dtype=torch.float64) for t in (x, a, b))
    for got, v, d in (
            (r.view(r.dx, 40), vx, loss(x + vx, a, b) - loss(x, a, b)),
            (r.da, va, loss(x, a + va, b) - loss(x, a, b)),
            (r.db, vb, loss(x, a, b + vb) - loss(x, a, b))):
        terms = got.double().cpu() * v
        # each gradient is a sum of at most 40 x 30 fp32 products, chained by 100
        assert abs(terms.sum() - d) <= 100 * U * 40 * terms.abs().sum()


@pytest.mark.parametrize("form", [(40, 640, 128, 16, 5), (700, 256, 320, 16, 5)], ids=str)
def test_repeats_are_identical_and_calls_overlap(form):
    rs = [Rows(*form, seed=s) for s in (1, 2)]
    for r in rs:
        r.forward()
        r.backward()
    want = [[t.clone() for t in (r.y, r.dx, r.da, r.db)] for r in rs]
    streams = [torch.cuda.Stream() for _ in range(2)]
    other = [torch.empty_like(r.ws) for r in rs]  # a call's own workspace
    torch.cuda.synchronize()
    for _ in range(3):
        for r, s, ws in zip(rs, streams, other):
            r.forward(stream=s)
            r.backward(stream=s)
    torch.cuda.synchronize()
    for r, w in zip(rs, want):
        for t, v in zip((r.y, r.dx, r.da, r.db), w):
            assert torch.equal(t, v)


@pytest.mark.parametrize("form", [(40, 640, 128, 16, 5), (700, 256, 320, 16, 5)], ids=str)
def test_captured_and_replayed(form):
    r = Rows(*form, live=form[0])
    r.forward()
    r.backward()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r.forward()
        r.backward()
    for seed in range(3):
        o = Rows(*form, seed=seed + 10)
        for t, v in ((r.x, o.x), (r.dy, o.dy), (r.ids, o.ids), (r.a, o.a)):
            t.copy_(v)
        r.count.fill_(form[0] - 3 * seed)
        for t in (r.y, r.dx, r.da, r.db):
            t.fill_(SENTINEL)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (r.y, r.dx, r.da, r.db)]
        for t in (r.y, r.dx, r.da, r.db):
            t.fill_(SENTINEL)
        r.forward()
        r.backward()
        torch.cuda.synchronize()
        for t, v in zip((r.y, r.dx, r.da, r.db), got):
            assert torch.equal(t, v)


def test_offsets_beyond_32_bits():
    """Two rows 2^31 elements apart, and adapters that reach beyond 2^31."""
    stride = 2 ** 31
    r = Rows(2, 64, 32, 4, 2, order="last")
    r.forward()
    x = torch.empty(stride + 64, dtype=torch.bfloat16, device="cuda")
    y = torch.empty(stride + 32, dtype=torch.bfloat16, device="cuda")
    for i in range(2):
        x[i * stride:i * stride + 64] = r.view(r.x, 64)[i]
    d = nsc.make_adapter_desc(64, 32, 4, 2, dtype=nsc.NSC_T_BF16, x_stride=stride, y_stride=stride)
    nsc.nsc_adapter_project(d, x, r.w, r.bias, r.a, r.b, r.scale, r.ids, y, r.ws, 2)
    for i in range(2):
        assert torch.equal(y[i * stride:i * stride + 32], r.view(r.y, 32)[i])
    del x, y
    m, rank, k = 35000, 64, 1024  # 2.3e9 elements of a
    small = Rows(3, k, 16, rank, 1, order="last")
    a = torch.empty((m, rank * k), dtype=torch.bfloat16, device="cuda")
    b = torch.empty((m, 16 * rank), dtype=torch.bfloat16, device="cuda")
    a[-1], b[-1] = small.a, small.b
    scale = torch.full((m,), small.scale.item(), device="cuda")
    ids = torch.full((3,), m - 1, dtype=torch.int32, device="cuda")
    d = nsc.make_adapter_desc(k, 16, rank, m, dtype=nsc.NSC_T_BF16)
    y = torch.empty(48, dtype=torch.bfloat16, device="cuda")
    nsc.nsc_adapter_project(d, small.x, small.w, small.bias, a, b, scale, ids, y, small.ws, 3)
    small.forward()
    assert torch.equal(y, small.y)

"""GPU tests of nsc_group_norm and nsc_group_norm_backward against fp64."""
import math

import pytest
import torch

import paper_1703_02529_amd as nsc

pytestmark = pytest.mark.gpu

TYPES = {"f32": (nsc.NSC_T_F32, torch.float32), "bf16": (nsc.NSC_T_BF16, torch.bfloat16),
         "f16": (nsc.NSC_T_F16, torch.float16)}
ACTS = {"none": nsc.NSC_ACT_NONE, "relu": nsc.NSC_ACT_RELU, "silu": nsc.NSC_ACT_SILU}
U = 2.0 ** -24   # half a step of fp32
EPS = 1e-5
SENTINEL = 7.0


class Maps:
    """One call's buffers: n images, `pad` elements apart, `shift` elements off
    the allocation's start, `live` of them counted on the device (None: no
    count is passed)."""

    def __init__(self, n, h, w, c, groups, dtype="bf16", act="relu", pad=0, shift=0, live=None,
                 seed=0, mean=0.5, fill=None):
        self.n, self.hw, self.c, self.g, self.act = n, h * w, c, groups, act
        code, self.t = TYPES[dtype]
        self.live = n if live is None else min(max(live, 0), n)
        e = h * w * c
        self.stride = e + pad
        g = torch.Generator().manual_seed(seed)
        x = torch.randn((n, h * w, c), generator=g, dtype=torch.float64)
        x = x * (torch.rand(c, generator=g) + 0.3) + mean * torch.randn(c, generator=g)
        if fill is not None:
            x = fill(x)
        self.x = self._dev(x.reshape(n, e), shift, pad)
        self.dy = self._dev(torch.randn((n, e), generator=g, dtype=torch.float64), shift, pad)
        self.gamma = (1 + 0.3 * torch.randn(c, generator=g)).cuda()
        self.beta = (0.4 * torch.randn(c, generator=g)).cuda()
        self.y = torch.full_like(self.x, SENTINEL)
        self.dx = torch.full_like(self.x, SENTINEL)
        self.stats = torch.full((n, groups, 2), SENTINEL, device="cuda")
        self.dgamma = torch.full((c,), SENTINEL, device="cuda")
        self.dbeta = torch.full((c,), SENTINEL, device="cuda")
        self.count = None if live is None else torch.tensor([live], dtype=torch.int32).cuda()
        self.desc = nsc.make_norm_desc(h, w, c, groups, act=ACTS[act], dtype=code, eps=EPS,
                                       x_stride=self.stride, y_stride=self.stride)
        size = max(nsc.nsc_group_norm_workspace_bytes(self.desc, n, backward=b) for b in (0, 1))
        self.ws = torch.empty(max(256, size), dtype=torch.uint8, device="cuda")

    def _dev(self, v, shift, pad):
        n, e = v.shape
        buf = torch.full((shift + n * (e + pad),), SENTINEL, dtype=self.t, device="cuda")
        rows = buf[shift:]
        rows.view(n, e + pad)[:, :e] = v.cuda().to(self.t)
        return rows

    def rows(self, buf):
        return buf.view(self.n, self.stride)[:, :self.hw * self.c]

    def forward(self, stats=True, stream=None, y=None):
        nsc.nsc_group_norm(self.desc, self.x, self.gamma, self.beta, self.y if y is None else y,
                           self.ws, self.n, stats=self.stats if stats else None, count=self.count,
                           stream=stream)

    def backward(self, stream=None):
        nsc.nsc_group_norm_backward(self.desc, self.x, self.dy, self.gamma, self.beta, self.stats,
                                    self.dx, self.dgamma, self.dbeta, self.ws, self.n,
                                    count=self.count, stream=stream)

    def maps64(self, buf):
        return self.rows(buf)[:self.live].double().cpu().view(self.live, self.hw, self.c)

    def reference(self, x=None):
        """fp64 (mean, rstd, xh, z, y), per-channel shapes [live, hw, c]."""
        x = self.maps64(self.x) if x is None else x
        cpg = self.c // self.g
        v = x.view(self.live, self.hw, self.g, cpg)
        mean = v.mean((1, 3))
        var = ((v - mean[:, None, :, None]) ** 2).mean((1, 3))
        rstd = 1 / torch.sqrt(var + EPS)
        wide = lambda s: s.repeat_interleave(cpg, 1)[:, None, :]
        xh = (x - wide(mean)) * wide(rstd)
        z = xh * self.gamma.double().cpu() + self.beta.double().cpu()
        y = {"none": z, "relu": z.clamp(min=0), "silu": z * torch.sigmoid(z)}[self.act]
        return mean, rstd, wide(mean), wide(rstd), xh, z, y


def levels(m):
    """Most fp32 roundings one after another in a statistic, by any order the
    kernels use: a thread's own pixels (at most 2^24 / 64 joined eight at a
    time, a chunk's 64 values one by one), then a group's threads (1024 x 8
    entries dealt over 64 lanes, 6 shuffle steps), then up to 64 parts."""
    return 64 + 4 * math.ceil(m.hw / 8) / 4 + 128 + 6 + 64


def check_forward(m):
    half = torch.finfo(m.t).eps / 2
    mean, rstd, wmean, wrstd, xh, z, y = m.reference()
    got = m.maps64(m.y)
    L = levels(m) * U
    x = m.maps64(m.x)
    v = x.view(m.live, m.hw, m.g, m.c // m.g)
    top = v.abs().amax((1, 3))
    got_stats = m.stats[:m.live].double().cpu()
    assert ((got_stats[..., 0] - mean).abs() <= L * top).all()
    # the variance's terms are squares: L relative, and the mean's error twice;
    # rstd takes half of it, its square root and division two roundings
    rel = 2 * L + (L * top * rstd) ** 2 + 2 * L * top * rstd + 4 * U
    assert ((got_stats[..., 1] - rstd).abs() <= rel * rstd).all()
    wide = lambda s: s.repeat_interleave(m.c // m.g, 1)[:, None, :]
    ga = m.gamma.double().cpu().abs()
    # z = (x - mean) * (gamma rstd) + beta: the mean's error, rstd's, five roundings
    dz = ga * wrstd * L * wide(top) + (wide(rel) + 5 * U) * (ga * xh.abs()) + U * z.abs()
    # SiLU's slope is at most 1.1; its exp, add, reciprocal and product, and exp's
    # argument (|z| U absolute, for z of either sign)
    tol = half * y.abs() + (1 + half) * (1.1 * dz + (8 + z.abs()) * U * y.abs())
    tol += 2.0 ** -25 if m.t == torch.float16 else 0  # half a step of the smallest fp16 values
    bad = (got - y).abs() > tol
    assert not bad.any(), (bad.sum().item(), ((got - y).abs() - tol).max().item())


def untouched(m, buf):
    """Images behind the count and the gaps between images hold what they held."""
    full = buf.view(m.n, m.stride).float().cpu()
    assert (full[m.live:] == SENTINEL).all()
    assert (full[:, m.hw * m.c:] == SENTINEL).all()


FORMS = [  # n, h, w, c, groups
    (3, 25, 25, 32, 8), (2, 50, 50, 64, 8), (5, 12, 12, 64, 1), (4, 12, 12, 64, 64),
    (1, 1, 1, 16, 4), (2, 1, 1, 5, 5), (3, 2, 1, 3, 1), (2, 7, 5, 45, 5), (2, 9, 9, 40, 4),
    (1, 3, 3, 24, 2), (2, 5, 4, 72, 8), (1, 4, 4, 1024, 1), (1, 2, 3, 2040, 2040),
    (1, 3, 2, 1021, 1021), (2, 17, 3, 96, 3), (1, 112, 112, 40, 4), (2, 60, 60, 320, 32),
    (300, 6, 6, 16, 2), (1, 200, 300, 8, 1), (1, 100, 100, 17, 1),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("form", FORMS, ids=str)
def test_forward(form, dtype):
    act = ("none", "relu", "silu")[sum(form) % 3]
    m = Maps(*form, dtype=dtype, act=act)
    m.forward()
    check_forward(m)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad,shift", [(8, 0), (3, 0), (0, 1), (8, 8), (1, 5)])
@pytest.mark.parametrize("live", [None, 0, 1, 3, 4, 9, -2])
def test_strides_alignment_and_counts(dtype, pad, shift, live):
    m = Maps(4, 10, 9, 32, 4, dtype=dtype, act="silu", pad=pad, shift=shift, live=live)
    m.forward()
    check_forward(m)
    untouched(m, m.y)
    assert (m.stats[m.live:] == SENTINEL).all()
    m.backward()
    check_backward(m)
    untouched(m, m.dx)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("form", [(2, 3, 3, 1024, 1), (1, 40, 40, 700, 1), (3, 2, 2, 1023, 1)],
                         ids=str)
def test_wide_groups_off_every_alignment(form, dtype):
    """Groups of more channels than half a workgroup, one element at a time."""
    m = Maps(*form, dtype=dtype, act="relu", pad=1, shift=1)
    m.forward()
    check_forward(m)
    untouched(m, m.y)
    m.backward()
    check_backward(m)
    untouched(m, m.dx)


def test_in_place_and_without_statistics():
    m = Maps(6, 30, 30, 64, 8)
    m.forward()
    x = m.x.clone()
    m.forward(stats=False, y=m.x)
    assert torch.equal(m.x, m.y) and not torch.equal(m.x, x)


@pytest.mark.parametrize("value", [0.0, 3.0, -1e4])
@pytest.mark.parametrize("form", [(2, 12, 12, 64, 8), (1, 112, 112, 64, 8), (2, 5, 5, 15, 3)],
                         ids=str)
def test_constant_maps(value, form):
    """Variance 0: y is act(beta) up to what eps leaves of the mean's rounding."""
    m = Maps(*form, dtype="f32", act="none", fill=lambda x: x * 0 + value)
    m.forward()
    check_forward(m)
    m.backward()
    check_backward(m)


@pytest.mark.parametrize("form", [(3, 25, 25, 64, 8), (1, 90, 90, 64, 4)], ids=str)
def test_far_means(form):
    """A mean of 1,000 deviations: no square of the mean enters the variance."""
    m = Maps(*form, dtype="f32", act="none", fill=lambda x: x + 1000)
    m.forward()
    check_forward(m)


@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_not_a_number_stays_in_its_group(value):
    m = Maps(3, 20, 20, 64, 8, act="relu")
    m.forward()
    m.backward()
    y, dx, stats = m.y.clone(), m.dx.clone(), m.stats.clone()
    m.rows(m.x)[1, 5 * 64 + 17] = value  # image 1, group 2
    m.forward()
    hit = torch.zeros((3, 400, 64), dtype=torch.bool, device="cuda")
    hit[1, :, 16:24] = True
    hit = hit.view(3, -1)
    assert torch.equal(m.rows(m.y)[~hit], m.rows(y)[~hit])
    assert torch.isnan(m.rows(m.y).float()[hit]).all()
    keep = torch.ones((3, 8), dtype=torch.bool, device="cuda")
    keep[1, 2] = False
    assert torch.equal(m.stats[keep], stats[keep])
    m.stats.copy_(stats)  # finite statistics beside an infinite value
    m.backward()
    assert torch.equal(m.rows(m.dx)[~hit], m.rows(dx)[~hit])


def grads64(m):
    """Gradients by the formula in fp64, from the statistics the kernel got."""
    x, dy = m.maps64(m.x), m.maps64(m.dy)
    cpg, k = m.c // m.g, m.c // m.g * m.hw
    st = m.stats[:m.live].double().cpu().repeat_interleave(cpg, 1)[:, None, :, :]
    mean, rstd = st[..., 0], st[..., 1]
    ga, be = m.gamma.double().cpu(), m.beta.double().cpu()
    xh = (x - mean) * rstd
    z = xh * ga + be
    s = torch.sigmoid(z)
    slope = {"none": torch.ones_like(z), "relu": (z > 0).double(),
             "silu": s * (1 + z * (1 - s))}[m.act]
    dz = dy * slope
    grouped = lambda v: v.view(m.live, m.hw, m.g, cpg).sum((1, 3)).repeat_interleave(
        cpg, 1)[:, None, :] / k
    dx = rstd * (ga * dz - grouped(ga * dz) - xh * grouped(ga * dz * xh))
    # the magnitudes of the terms: of dz with the rounding of its slope, and of dx
    dslope = 0.0 if m.act != "silu" else 0.5 * 4 * U * (xh.abs() * ga.abs() + be.abs()) + 16 * U * (
        1 + z.abs())
    err = dy.abs() * dslope + 4 * U * dz.abs()
    t1, t2 = (ga * dz).abs(), (ga * dz * xh).abs()
    K = levels(m) + m.hw  # a thread's pixels one by one
    e1 = ga.abs() * err
    tol = rstd * (e1 + grouped(e1) + xh.abs() * grouped(e1 * xh.abs()) + 8 * U * t1 +
                  (K + 8) * U * (grouped(t1) + xh.abs() * grouped(t2)))
    pg = ((dz * xh).sum((0, 1)), ((K + 8) * U * (dz * xh).abs() + err * xh.abs()).sum((0, 1)))
    pb = (dz.sum((0, 1)), ((K + 8) * U * dz.abs() + err).sum((0, 1)))
    return dx, tol, pg, pb


def check_backward(m):
    half = torch.finfo(m.t).eps / 2
    dx, tol, (dgamma, tg), (dbeta, tb) = grads64(m)
    got = m.maps64(m.dx)
    tol = (1 + half) * tol + half * dx.abs() + (2.0 ** -25 if m.t == torch.float16 else 0)
    assert not ((got - dx).abs() > tol).any(), ((got - dx).abs() - tol).max().item()
    assert ((m.dgamma.double().cpu() - dgamma).abs() <= tg + U * dgamma.abs()).all()
    assert ((m.dbeta.double().cpu() - dbeta).abs() <= tb + U * dbeta.abs()).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("form", FORMS, ids=str)
def test_backward(form, dtype):
    act = ("silu", "none", "relu")[sum(form) % 3]
    m = Maps(*form, dtype=dtype, act=act)
    m.forward()
    m.backward()
    check_backward(m)


def test_relu_sign_next_to_zero():
    """x = mean exactly, and beta a step either side of zero: the slope is the
    exact value's."""
    m = Maps(1, 8, 8, 8, 1, dtype="f32", act="relu", fill=lambda x: torch.where(
        torch.arange(64)[:, None] % 2 == 0, 1.0, -1.0).expand_as(x))
    m.beta.copy_(torch.tensor([0.0, 1e-30, -1e-30, 0.0, 1.0, -1.0, 0.5, -0.5]))
    m.gamma.copy_(torch.tensor([0.0, 0.0, 0.0, 1.0, -1.0, 1.0, 1.0, 1.0]))
    m.forward()
    st = m.stats.double().cpu()
    # |z| below a rounding: beta cancels the last channels' gamma xh to the last bit
    xh = ((1.0 - st[0, 0, 0]) * st[0, 0, 1]).item()
    m.beta[4:8] = torch.tensor([xh, -xh, -xh * (1 + 2.0 ** -23), -xh * (1 - 2.0 ** -24)])
    m.backward()
    check_backward(m)


def test_backward_against_differences():
    """The gradient along a direction against a central difference of the fp64
    forward pass (the statistics move with x)."""
    m = Maps(2, 9, 7, 24, 4, dtype="f32", act="silu")
    m.forward()
    m.backward()
    g = torch.Generator().manual_seed(5)
    x, dy = m.maps64(m.x), m.maps64(m.dy)
    v = torch.randn(x.shape, generator=g, dtype=torch.float64)
    h = 1e-4  # the difference's own error: h^2 = 1e-8 of the third derivatives
    d = ((m.reference(x + h * v)[-1] - m.reference(x - h * v)[-1]) * dy).sum() / (2 * h)
    got = (m.maps64(m.dx) * v).sum()
    scale = (m.maps64(m.dx) * v).abs().sum()
    assert abs(got - d) <= 1e-6 * scale
    for grad, p in ((m.dgamma, m.gamma), (m.dbeta, m.beta)):
        keep, u = p.clone(), torch.randn(24, generator=g).cuda()
        ys = []
        for sign in (1, -1):
            p.copy_(keep + sign * 2.0 ** -10 * u)
            ys.append((m.reference(x)[-1] * dy).sum())
        p.copy_(keep)
        # each end of the step is rounded by 2^-24 of the parameter; the step's
        # square, (2^-10 x 10)^2, times the third derivative (at most 1 of the slope)
        tol = (grad.abs() * keep.abs()).sum().item() * 2.0 ** -14
        tol += 1e-4 * (grad * u).abs().sum().item()
        assert abs((ys[0] - ys[1]).item() * 2.0 ** 9 - (grad * u).sum().item()) <= tol


def test_no_images_leave_zero_parameter_gradients():
    for live, n in ((0, 3), (None, 0)):
        m = Maps(3, 4, 4, 16, 2, live=live)
        nsc.nsc_group_norm_backward(m.desc, m.x, m.dy, m.gamma, m.beta, m.stats, m.dx, m.dgamma,
                                    m.dbeta, m.ws, n, count=m.count)
        assert (m.dgamma == 0).all() and (m.dbeta == 0).all()
        assert (m.dx == SENTINEL).all()


@pytest.mark.parametrize("form", [(40, 25, 25, 64, 8), (1, 112, 112, 64, 8)], ids=str)
def test_repeats_are_identical_and_calls_overlap(form):
    """The same bits on every run, on two streams at once with a workspace each."""
    a, b = Maps(*form, seed=1), Maps(*form, seed=2)
    for m in (a, b):
        m.forward()
        m.backward()
    want = [(m.y.clone(), m.dx.clone(), m.dgamma.clone(), m.dbeta.clone()) for m in (a, b)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(3):
        for m, s in zip((a, b), streams):
            m.forward(stream=s)
            m.backward(stream=s)
    torch.cuda.synchronize()
    for m, w in zip((a, b), want):
        for got, exp in zip((m.y, m.dx, m.dgamma, m.dbeta), w):
            assert torch.equal(got, exp)


@pytest.mark.parametrize("form", [(40, 25, 25, 64, 8), (1, 112, 112, 64, 8)], ids=str)
def test_captured_and_replayed(form):
    m = Maps(*form, live=form[0])
    m.forward()
    m.backward()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        m.forward()
        m.backward()
    for seed in range(3):
        other = Maps(*form, seed=seed + 10)
        m.x.copy_(other.x)
        m.dy.copy_(other.dy)
        m.count.fill_(form[0] - (seed == 1))
        m.y.fill_(SENTINEL)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (m.y, m.dx, m.dgamma, m.dbeta)]
        m.y.fill_(SENTINEL)
        m.forward()
        m.backward()
        torch.cuda.synchronize()
        for g, e in zip(got, (m.y, m.dx, m.dgamma, m.dbeta)):
            assert torch.equal(g, e)


def test_offsets_beyond_32_bits():
    """Images 2^31 + 8 elements apart."""
    stride = 2 ** 31 + 8
    n, h, w, c = 2, 6, 6, 16
    e = h * w * c
    x = torch.empty(stride + e, dtype=torch.bfloat16, device="cuda")
    y = torch.empty_like(x)
    small = Maps(n, h, w, c, 4)
    for i in range(n):
        x[i * stride:i * stride + e] = small.rows(small.x)[i]
    d = nsc.make_norm_desc(h, w, c, 4, act=ACTS["relu"], dtype=nsc.NSC_T_BF16, eps=EPS,
                           x_stride=stride, y_stride=stride)
    nsc.nsc_group_norm(d, x, small.gamma, small.beta, y, small.ws, n)
    small.forward()
    for i in range(n):
        assert torch.equal(y[i * stride:i * stride + e], small.rows(small.y)[i])

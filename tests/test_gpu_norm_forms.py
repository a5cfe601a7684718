"""GPU tests of nsc_group_norm and nsc_group_norm_backward by every kernel that
their plan picks (layer_forms.py): each value counted once, and each result to
the roundings of its own formula."""
import pytest
import torch

import paper_1703_02529_amd as nsc
from layer_forms import norm_forms
from test_gpu_norm import ACTS, EPS, SENTINEL, TYPES, U, Maps

pytestmark = pytest.mark.gpu
DEV = "cuda"


class Images:
    """Buffers of one call; values are made and checked on the GPU."""

    def __init__(self, dtype, n, hw, c, groups, pad, act, seed=0):
        self.n, self.hw, self.c, self.g, self.act = n, hw, c, groups, act
        code, self.t = TYPES[dtype]
        self.e, self.stride = hw * c, hw * c + pad
        self.gen = torch.Generator(device=DEV).manual_seed(seed)
        self.desc = nsc.make_norm_desc(1, hw, c, groups, act=ACTS[act], dtype=code, eps=EPS,
                                       x_stride=self.stride, y_stride=self.stride)
        self.gamma, self.beta = torch.ones(c, device=DEV), torch.zeros(c, device=DEV)
        self.stats = torch.full((n, groups, 2), SENTINEL, device=DEV)
        size = max(nsc.nsc_group_norm_workspace_bytes(self.desc, n, backward=b) for b in (0, 1))
        self.ws = torch.empty(max(256, size), dtype=torch.uint8, device=DEV)

    def buffer(self, values=None):
        buf = torch.full((self.n, self.stride), SENTINEL, dtype=self.t, device=DEV)
        if values is not None:
            buf[:, :self.e] = values.reshape(self.n, self.e)
        return buf

    def ints(self, low, high):
        return torch.randint(low, high + 1, (self.n, self.e), generator=self.gen, device=DEV,
                             dtype=torch.int8)

    def maps(self, buf):
        return buf[:, :self.e].view(self.n, self.hw, self.c)

    def per_channel(self, per_group):
        """[n, groups] as [n, 1, c]."""
        return per_group.repeat_interleave(self.c // self.g, 1)[:, None, :]

    def forward(self, x, y):
        nsc.nsc_group_norm(self.desc, x, self.gamma, self.beta, y, self.ws, self.n,
                           stats=self.stats)


def _id(form):
    return "-".join(map(str, form))


@pytest.mark.parametrize("form", norm_forms(False), ids=_id)
def test_forward(form):
    m = Images(*form, act=("none", "relu", "silu")[form[2] % 3])
    c, half = m.c, torch.finfo(m.t).eps / 2
    m.gamma = 1 + 0.3 * torch.randn(c, generator=m.gen, device=DEV)
    m.beta = 0.4 * torch.randn(c, generator=m.gen, device=DEV)
    v = torch.randn((m.n, m.hw, c), generator=m.gen, device=DEV)
    v = v * (torch.rand(c, generator=m.gen, device=DEV) + 0.3)
    x, y = m.buffer(v + 0.5 * torch.randn(c, generator=m.gen, device=DEV)), m.buffer()
    del v
    m.forward(x, y)
    assert (y[:, m.e:] == SENTINEL).all()
    # the statistics: at most 320 roundings one after another (a thread's 160 values
    # and the joins of its chunks, its group's lanes, the parts)
    cpg, f = c // m.g, m.maps(x).double()
    grouped = f.view(m.n, m.hw, m.g, cpg)
    mean = grouped.mean((1, 3))
    var = ((grouped - mean[:, None, :, None]) ** 2).mean((1, 3))
    got_mean, got_rstd = m.stats.double().unbind(2)
    top = grouped.abs().amax((1, 3))
    assert ((got_mean - mean).abs() <= 320 * U * top).all()
    rstd = 1 / torch.sqrt(var + EPS)
    assert ((got_rstd - rstd).abs() <= (2 * 320 * U * (1 + top * rstd) + 4 * U) * rstd).all()
    del grouped
    # the result, from the kernel's own statistics: the difference, gamma rstd and the
    # fused product and sum are rounded; the activation as in test_gpu_norm.py
    p = (f - m.per_channel(got_mean)) * (m.per_channel(got_rstd) * m.gamma.double())
    z = p + m.beta.double()
    del f
    want = {"none": z, "relu": z.clamp(min=0), "silu": z * torch.sigmoid(z)}[m.act]
    tol = 1.1 * (2 * U * p.abs() + U * z.abs()) * (1 + half) + half * want.abs()
    if m.act == "silu":
        tol += (1 + half) * (8 + z.abs()) * U * want.abs()
    tol += 2.0 ** -25 if m.t == torch.float16 else 1e-37  # the smallest values' half step
    over = (m.maps(y).double() - want).abs() - tol
    assert not (over > 0).any(), over.max().item()
    # in place
    m.forward(x, x)
    assert torch.equal(x, y)


@pytest.mark.parametrize("form", norm_forms(False), ids=_id)
def test_every_value_counts_once(form):
    """Maps of zeros with one value 2^k per group, at another place in each image and
    group, the first and the last among them: the mean is that value over the
    count, which sums with zeros keep to a few roundings, and half or twice of it
    would be a value left out or taken twice."""
    m = Images(*form, act="none")
    cpg = m.c // m.g
    count, value = m.hw * cpg, 2.0 ** 10
    for turn in range(1 if m.n * m.g > 1000 else 24):
        at = torch.linspace(0, count - 1, m.n * m.g, device=DEV, dtype=torch.float64).long()
        if turn:  # few images are split: both sides of the parts' ends, however many
            ends = torch.randint(0, 65, at.shape, generator=m.gen, device=DEV) * m.hw // 64
            pixel = ends - torch.randint(0, 2, at.shape, generator=m.gen, device=DEV)
            at = pixel.clamp(0, m.hw - 1) * cpg + torch.randint(0, cpg, at.shape, generator=m.gen,
                                                                device=DEV)
        v = torch.zeros((m.n, m.g, m.hw, cpg), dtype=m.t, device=DEV)
        v.view(m.n * m.g, count).scatter_(1, at[:, None], value)
        v = v.transpose(1, 2).contiguous()
        x = m.buffer(v)
        m.forward(x, m.buffer())
        mean, rstd = m.stats.double().unbind(2)
        # each chunk and part is joined by four roundings, up to 80 of them
        assert ((mean - value / count).abs() <= 320 * U * value / count).all()
        var = (value / count) * value * (1 - 1 / count)
        want = (var + EPS) ** -0.5
        assert ((rstd - want).abs() <= 2 * 320 * U * want).all()


@pytest.mark.parametrize("form", norm_forms(True), ids=_id)
def test_backward_of_whole_numbers(form):
    """x and dy are small whole numbers, gamma is 1, 2 or -1 and the statistics are
    (0, 1): xh = x, every sum is exact in any order, and dbeta and dgamma must be
    equal.  With ReLU, beta = 1/2 and gamma 1 or 2 leave dy where x >= 0."""
    m = Images(*form, act=("none", "relu")[form[2] % 2])
    c, half = m.c, torch.finfo(m.t).eps / 2
    x, dy = m.buffer(m.ints(-3, 3)), m.buffer(m.ints(-4, 4))
    dx = m.buffer()
    m.gamma = (torch.tensor([1.0, 2.0, 1.0]) if m.act == "relu" else
               torch.tensor([1.0, 2.0, -1.0])).repeat(c)[:c].to(DEV)
    m.beta = torch.full((c,), 0.5, device=DEV)
    m.stats.copy_(torch.tensor([0.0, 1.0]))
    dgamma, dbeta = (torch.full((c,), SENTINEL, device=DEV) for _ in range(2))
    nsc.nsc_group_norm_backward(m.desc, x, dy, m.gamma, m.beta, m.stats, dx, dgamma, dbeta, m.ws,
                                m.n)
    xh, dz = m.maps(x).double(), m.maps(dy).double()
    if m.act == "relu":
        dz = dz * (xh >= 0)
    assert torch.equal(dbeta.double(), dz.sum((0, 1)))
    assert torch.equal(dgamma.double(), (dz * xh).sum((0, 1)))
    q = dz * m.gamma.double()
    group = lambda v: m.per_channel(v.view(m.n, m.hw, m.g, c // m.g).mean((1, 3)))
    m1, m2 = group(q), group(q * xh)
    want = q - m1 - xh * m2
    # each mean: the count's reciprocal and the product; then the two fused products
    tol = 4 * U * (m1.abs() + (xh * m2).abs()) + 2 * U * want.abs()
    tol = (1 + half) * tol + half * want.abs() + 2.0 ** -25 * (m.t == torch.float16)
    over = (m.maps(dx).double() - want).abs() - tol
    assert not (over > 0).any(), over.max().item()
    assert (dx[:, m.e:] == SENTINEL).all()


@pytest.mark.parametrize("form", [(40, 25, 25, 64, 8), (1, 112, 112, 64, 8)], ids=str)
def test_overlapping_calls_write_everything(form):
    """Two calls on two streams, each with its own workspace, into outputs that
    were cleared before."""
    ms = [Maps(*form, seed=s) for s in (1, 2)]
    outs = [(m.y, m.stats, m.dx, m.dgamma, m.dbeta) for m in ms]
    for m in ms:
        m.forward()
        m.backward()
    want = [[t.clone() for t in o] for o in outs]
    streams = [torch.cuda.Stream() for _ in ms]
    for _ in range(3):
        for o in outs:
            for t in o:
                t.fill_(SENTINEL)
        torch.cuda.synchronize()
        for m, s in zip(ms, streams):
            m.forward(stream=s)
            m.backward(stream=s)
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            assert all(torch.equal(t, v) for t, v in zip(o, w))

"""GPU tests of nsc_group_norm and nsc_group_norm_backward at their largest:
maps of more than 2^31 values,
more blocks of images than a launch holds workgroups."""
import math

import pytest
import torch

import paper_1703_02529_amd as nsc

pytestmark = pytest.mark.gpu
DEV = "cuda"


def test_a_map_of_more_than_2_31_values():
    """4096 x 4096 x 129 in 3 groups (channels that fill no vectors), with values
    at which every sum is exact: x = 1 on even pixels and -1 on odd ones, dy =
    x + 1, gamma = 1, beta = 0, and the statistics (0, 1/2) that make xh = x / 2.
    Then dbeta = hw, dgamma = hw / 2, the group's means are m1 = 1 and m2 = 1/2,
    and dx = (dy - 1 - x / 4) / 2 = 3/8 x.  (1 / (hw cpg) is rounded, 2^-24, far
    below bf16's half step.)"""
    hw, c, groups = 4096 * 4096, 129, 3
    x = torch.ones((hw, c), dtype=torch.bfloat16, device=DEV)
    x[1::2] = -1
    dy = x + 1
    out = torch.full_like(x, 7)
    gamma, beta = torch.ones(c, device=DEV), torch.zeros(c, device=DEV)
    dgamma, dbeta = torch.zeros(c, device=DEV), torch.zeros(c, device=DEV)
    d = nsc.make_norm_desc(4096, 4096, c, groups, dtype=nsc.NSC_T_BF16, eps=1e-5)
    size = max(nsc.nsc_group_norm_workspace_bytes(d, 1, backward=b) for b in (0, 1))
    ws = torch.empty(max(256, size), dtype=torch.uint8, device=DEV)
    stats = torch.tensor([0.0, 0.5], device=DEV).repeat(groups)
    nsc.nsc_group_norm_backward(d, x, dy, gamma, beta, stats, out, dgamma, dbeta, ws, 1)
    assert (dbeta == hw).all(), dbeta
    assert (dgamma == hw / 2).all(), dgamma
    assert torch.equal(out, x * 0.375)
    # forward: mean 0 and variance 1 exactly, rstd and y each rounded
    nsc.nsc_group_norm(d, x, gamma, beta, out, ws, 1, stats=stats)
    rstd = 1 / math.sqrt(1 + d.eps)
    got = stats.view(groups, 2).double().cpu()
    assert (got[:, 0] == 0).all() and ((got[:, 1] - rstd).abs() <= 3 * 2.0 ** -24).all()
    assert torch.equal(out, x * torch.tensor(rstd, dtype=torch.bfloat16, device=DEV))


def test_more_blocks_than_a_launch_has_workgroups():
    """262,200 images in 64 blocks each are 16,780,800, and a launch of workgroups
    of 256 threads holds 2^24 - 1: workgroups take further blocks.  Every image
    as in a call of fewer, which are launched whole."""
    n, c, groups, part = 262200, 4096, 64, 65550
    g = torch.Generator(device=DEV).manual_seed(3)
    x = torch.randn((n, c), generator=g, device=DEV, dtype=torch.bfloat16)
    dy = torch.randint(-4, 5, (n, c), generator=g, device=DEV, dtype=torch.int8).bfloat16()
    gamma = 1 + 0.3 * torch.randn(c, generator=g, device=DEV)
    beta = 0.3 * torch.randn(c, generator=g, device=DEV)
    d = nsc.make_norm_desc(1, 1, c, groups, dtype=nsc.NSC_T_BF16)
    size = max(nsc.nsc_group_norm_workspace_bytes(d, n, backward=b) for b in (0, 1))
    ws = torch.empty(max(256, size), dtype=torch.uint8, device=DEV)

    def run(at, m):
        y, dx = (torch.full((m, c), 7.0, device=DEV, dtype=torch.bfloat16) for _ in range(2))
        stats = torch.zeros((m, groups, 2), device=DEV)
        dgamma, dbeta = torch.zeros(c, device=DEV), torch.zeros(c, device=DEV)
        nsc.nsc_group_norm(d, x[at:at + m], gamma, beta, y, ws, m, stats=stats)
        nsc.nsc_group_norm_backward(d, x[at:at + m], dy[at:at + m], gamma, beta, stats, dx, dgamma,
                                    dbeta, ws, m)
        return y, dx, stats, dgamma, dbeta

    y, dx, stats, dgamma, dbeta = run(0, n)
    dg, mag = torch.zeros(c, dtype=torch.float64, device=DEV), 0.0
    for at in range(0, n, part):
        few = run(at, part)
        for whole, some in zip((y, dx, stats), few):
            assert torch.equal(whole[at:at + part], some), at
        dg += few[3].double()
        mag = mag + few[3].double().abs()
    # sums of small whole numbers are exact; dgamma is rounded once here and per part there
    assert torch.equal(dbeta, dy.sum(0, dtype=torch.float64).float())
    assert ((dgamma.double() - dg).abs() <= 2.0 ** -24 * (mag + dg.abs())).all()


def test_room_for_the_most_images_and_a_few_of_them():
    """max_count = 2^31 - 1 with a count of 3: y = beta (variance 0), and what lies
    behind the count is left as it was."""
    n = 2 ** 31 - 1
    x = torch.empty(n, dtype=torch.bfloat16, device=DEV)
    y = torch.full((n,), 7.0, dtype=torch.bfloat16, device=DEV)
    x[:3] = torch.tensor([1.0, -2.0, 0.5])
    count = torch.tensor([3], dtype=torch.int32, device=DEV)
    d = nsc.make_norm_desc(1, 1, 1, 1, dtype=nsc.NSC_T_BF16)
    ws = torch.empty(max(256, nsc.nsc_group_norm_workspace_bytes(d, n)), dtype=torch.uint8,
                     device=DEV)
    nsc.nsc_group_norm(d, x, torch.ones(1, device=DEV), torch.full((1,), 0.25, device=DEV), y, ws,
                       n, count=count)
    assert (y[:3] == 0.25).all() and (y[3:] == 7).all()

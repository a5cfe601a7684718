"""GPU tests of nsc_group_norm and nsc_group_norm_backward at their largest:
maps of more than 2^31 values."""
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

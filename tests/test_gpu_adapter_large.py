"""GPU tests of nsc_adapter_project and nsc_adapter_backward at their largest:
more tiles, and more blocks of adapters, than a launch holds workgroups."""
import pytest
import torch

import paper_1703_02529_amd as nsc

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _ws(d, rows, backward=False):
    size = nsc.nsc_adapter_workspace_bytes(d, rows, backward=backward)
    return torch.empty(max(256, size), dtype=torch.uint8, device=DEV)


def test_more_blocks_of_adapters_than_a_launch_has_workgroups():
    """The most adapters, of 4,096 outputs each: b is transposed in 4,194,240
    blocks, beside 2,048 workgroups that list the rows, and a launch of workgroups
    of 1,024 threads holds 4,194,303.  Every used adapter has one row, so that its
    gradients are the products of that row in any order of the sums: they are
    those of a call that holds the used adapters alone."""
    m, n, k, d, rank = 65535, 300, 24, 4096, 1
    g = torch.Generator(device=DEV).manual_seed(1)
    r = lambda *s: torch.randn(s, generator=g, device=DEV, dtype=torch.bfloat16)
    x, dy, w = r(n, k), r(n, d), r(d, k)
    a, b = r(m, rank, k), r(m, d, rank)
    scale = torch.rand(m, generator=g, device=DEV) + 0.5
    used = torch.randperm(m - 1, generator=g, device=DEV)[:n - 1]
    ids = torch.cat([used, torch.tensor([m - 1], device=DEV)]).int()
    ids[7] = -1
    has = ids >= 0

    def run(desc, a, b, scale, ids):
        dx = torch.full((n, k), 7.0, dtype=torch.bfloat16, device=DEV)
        da = torch.full((desc.n_adapters, rank, k), 7.0, device=DEV)
        db = torch.full((desc.n_adapters, d, rank), 7.0, device=DEV)
        nsc.nsc_adapter_backward(desc, x, dy, w, a, b, scale, ids, dx, da, db,
                                 _ws(desc, n, True), n)
        return dx, da, db

    dx, da, db = run(nsc.make_adapter_desc(k, d, rank, m, dtype=nsc.NSC_T_BF16), a, b, scale, ids)
    at = ids[has].long()
    few = nsc.make_adapter_desc(k, d, rank, len(at), dtype=nsc.NSC_T_BF16)
    own = torch.full((n,), -1, dtype=torch.int32, device=DEV)
    own[has] = torch.arange(len(at), dtype=torch.int32, device=DEV)
    fx, fa, fb = run(few, a[at].contiguous(), b[at].contiguous(), scale[at].contiguous(), own)
    assert torch.equal(dx, fx) and torch.equal(da[at], fa) and torch.equal(db[at], fb)
    assert (fa != 0).any(2).all() and (fb != 0).any(1).all()
    da[at], db[at] = 0, 0
    assert not da.any() and not db.any()  # zeros for adapters without rows


def test_more_tiles_of_rows_than_a_launch_has_workgroups():
    """1,080,000,100 rows of one value are 16,875,002 tiles of 64, and a launch of
    workgroups of 256 threads holds 2^24 - 1.  Small whole numbers: every sum is
    exact."""
    n = 1_080_000_100
    d = nsc.make_adapter_desc(1, 1, 1, 1, dtype=nsc.NSC_T_BF16)
    x = (torch.arange(n, dtype=torch.int32, device=DEV) % 13).bfloat16()
    y = torch.full((n,), 99.0, dtype=torch.bfloat16, device=DEV)
    ids = torch.zeros(n, dtype=torch.int32, device=DEV)
    ids[5::7] = -1
    one = lambda v, t=torch.bfloat16: torch.full((1,), v, dtype=t, device=DEV)
    nsc.nsc_adapter_project(d, x, one(3.0), one(-2.0, torch.float32), one(2.0), one(1.0),
                            one(1.0, torch.float32), ids, y, _ws(d, n), n)
    # y = 3 x - 2, and 2 x more with the adapter
    x.mul_(3 + 2 * (ids == 0)).sub_(2)
    assert torch.equal(x, y)

"""GPU tests of nsc_group_norm and nsc_group_norm_backward at values where their
arithmetic could leave its range or its precision."""
import pytest
import torch

from test_gpu_norm import EPS, Maps

pytestmark = pytest.mark.gpu

# n, h, w, c, groups: in registers, split over workgroups, ragged vectors
VALUE_FORMS = [(3, 25, 25, 64, 8), (600, 30, 30, 64, 1), (1, 112, 112, 64, 8), (2, 7, 5, 45, 5),
               (1, 100, 100, 17, 1), (3, 4, 4, 20, 5)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("value", [2.0 ** 66, -2.0 ** 80])
@pytest.mark.parametrize("form", VALUE_FORMS, ids=str)
def test_constants_whose_square_overflows(form, value, dtype):
    """Powers of two: every sum of them and the mean are exact, the variance is 0
    and y is beta, although the mean's square is beyond fp32."""
    m = Maps(*form, dtype=dtype, act="none", fill=lambda x: x * 0 + value)
    m.forward()
    n, _, _, c, groups = form
    assert (m.stats[..., 0] == value).all()
    assert ((m.stats[..., 1].double() - EPS ** -0.5).abs() <= EPS ** -0.5 * 3 * 2.0 ** -24).all()
    assert torch.equal(m.rows(m.y).view(n, m.hw, c),
                       m.beta.to(m.t).expand(n, m.hw, c))

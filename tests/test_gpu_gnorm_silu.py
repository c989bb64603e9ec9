"""SiLU of the fp32 group norm over the whole range of its exponential.

Groups of equal values have x - mu = 0, so that u is beta exactly.  Tolerance, derived: u log2(e) is a product of two
rounded numbers (at most 1.3 x 2^-24 of itself), which the exponential turns into a relative error of |u| 2^-23 at most;
the exponential, the reciprocal, the sum and the last product add 2^-22, 2^-23 and twice 2^-24 (2^-21 in all); values of
the sigmoid below 2^-126 are zero."""
import numpy as np
import pytest
import torch

from gpu_util import to_np
from test_gpu_gnorm import u  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("most", [1.0, 20.0, 130.0])
def test_silu_far_out(u, most):  # noqa: F811
    beta = torch.linspace(-most, most, 8192, device="cuda")
    x = torch.full((64, 8192), 2.0, device="cuda")
    y, _, _ = u.ut_group_norm_fwd(x, None, beta, 32, act=u.UT_ACT_SILU)
    b = to_np(beta)
    ref = b / (1 + np.exp(-b))
    bound = np.abs(ref) * (2.0 ** -21 + np.where(b < 0, np.abs(b), 0) * 2.0 ** -23) + np.abs(b) * 2.0 ** -126
    err = np.abs(to_np(y) - ref)
    assert np.all(err <= bound), float((err / bound).max())

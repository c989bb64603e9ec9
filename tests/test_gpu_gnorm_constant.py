"""Group norm where a group's values are all equal: the mean is that value and x - mu is 0, so u is beta exactly.

Tolerance, derived: the activation carries 2^-20 of its value at |beta| < 2, the result is rounded once to bf16 (2^-8).
No term of the size of |mu| / sqrt(eps) may be left over, which for mu = 1000 and eps = 1e-6 is 10^6."""
import numpy as np
import pytest
import torch

from gpu_util import to_np
from test_gpu_gnorm import u  # noqa: F401

pytestmark = pytest.mark.gpu

ROUND = {torch.bfloat16: 2.0 ** -8, torch.float32: 0.0}


def constant(u, value, n, channels, groups, eps, act, dtype):  # noqa: F811
    g = torch.Generator().manual_seed(n + channels)
    gamma = (1 + 0.2 * torch.randn(channels, generator=g)).cuda()
    beta = (0.3 * torch.randn(channels, generator=g)).clamp(-1.9, 1.9).cuda()
    x = torch.full((n, channels), value, dtype=dtype, device="cuda")
    y, mean, rstd = u.ut_group_norm_fwd(x, gamma, beta, groups, eps=eps, act=act)
    assert torch.equal(mean, x[:1, :groups].float())
    assert np.allclose(to_np(rstd), eps ** -0.5, rtol=2.0 ** -22, atol=0)
    b = to_np(beta)
    ref = b / (1 + np.exp(-b)) if act else b
    assert np.all(np.abs(to_np(y) - ref) <= (ROUND[dtype] + 2.0 ** -20) * np.abs(ref))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("act", [0, 1])
@pytest.mark.parametrize("eps", [1e-5, 1e-6])
@pytest.mark.parametrize("value", [3.0, -100.0, 1000.0])
def test_constant_groups_give_beta(u, value, eps, act, dtype):  # noqa: F811
    constant(u, value, 64, 64, 8, eps, act, dtype)  # one block
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    constant(u, value, 32 * sms, 320, 32, eps, act, dtype)  # 32 rows a block


@pytest.mark.parametrize("value", [1000.0, -0.1, 3.0e5])
@pytest.mark.parametrize("rows", [3, 7, 23, 41, 47, 55, 61, 83, 97])
def test_constant_groups_over_many_blocks(u, rows, value):  # noqa: F811
    """Pieces of odd numbers of rows, some of one row more, merged over all blocks: the mean keeps every bit."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    for more in (0, sms // 2):
        constant(u, value, rows * sms + more, 1024, 32, 1e-5, 0, torch.float32)

"""The angles of the position rotation within the bounds that include/ultratex.h gives, against 60 decimal digits.

Tolerance, derived before the first run: heads whose pairs are all (1, 0) come out as sqrt(2) (cos a, sin a), so the
angle is that of the pair.  Sine and cosine are off by 2^-23 each, the products after them by 2^-24 of the value, which
turns the pair by 2^-22 at most, or 2^-24 turns; the header's bound comes on top."""
from decimal import Decimal, getcontext

import numpy as np
import pytest
import torch

from gpu_util import need_gpu, to_np

pytestmark = pytest.mark.gpu

PI = Decimal("3.14159265358979323846264338327950288419716939937510582097494459")
NEAR = [0, 1, 2, 77, 4095, 65537, 99991, 131071, 131072]
FAR = [16777217, 2 ** 30, 2 ** 30 + 12345, 2 ** 31 - 77, 2 ** 31 - 1]


@pytest.fixture(scope="module")
def u():
    need_gpu()
    from paper_2609_23169_gb300 import ultratex
    return ultratex


@pytest.mark.parametrize("theta", [1.0, 100.0, 1e4, 5e5, 0.5, 1e-3])
@pytest.mark.parametrize("axes", [(64, 0, 0), (0, 0, 64), (16, 24, 24)])
def test_angles(u, axes, theta):
    getcontext().prec = 60
    pos = NEAR + FAR
    side = 1 if axes[0] == 64 else 50000
    x = torch.zeros(len(pos), 1, 64, device="cuda")
    x[..., 0::2] = 1
    y = u.ut_qk_norm_rope_fwd(x, x, u.rope_config(side, axes, theta), eps=1e-12,
                              pos=torch.tensor(pos, dtype=torch.int32, device="cuda"))[0]
    y = to_np(y)[:, 0].astype(np.float64)
    got = np.arctan2(y[:, 1::2], y[:, 0::2]) / (2 * np.pi)
    theta = Decimal(float(np.float32(theta)))
    for i, p in enumerate(pos):
        at = (p // side ** 2, p % side ** 2 // side, p % side)
        e = 0
        for a in range(3):
            for j in range(axes[a] // 2):
                f = theta ** (Decimal(-2 * j) / axes[a]) / (2 * PI)
                off = (float((at[a] * f) % 1) - got[i, e] + 0.5) % 1 - 0.5
                bound = 2.0 ** (-25 if p <= 2 ** 17 else -20) + (float(at[a] * f) * 2.0 ** -46 if theta < 1 else 0.0)
                assert abs(off) <= bound + 2.0 ** -24, (p, a, j, off)
                e += 1

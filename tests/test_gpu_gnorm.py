"""Group norm with an activation, channels last, against the float64 oracle.

Tolerances (per element, derived, not fitted).  All arithmetic is fp32, each value rounded once: bf16 results are
within 2^-8 of themselves plus the fp32 error, fp32 results within the fp32 error alone.  fp32 error: the normalised
value (x - mu) r carries a few roundings of 2^-24 relative to |x| r + |xh| and the statistics' own error; sums of n
terms in two levels carry about n^(1/2) 2^-24 of their terms' magnitudes.  2^-17 of the terms' magnitudes covers both
for the sizes here with a factor of about 8 to spare."""
import numpy as np
import pytest
import torch

import oracle.conditioning_oracle as o
from gpu_util import need_gpu, to_np

pytestmark = pytest.mark.gpu

E = 2.0 ** -17
ROUND = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


@pytest.fixture(scope="module")
def u():
    need_gpu()
    from paper_2609_23169_gb300 import ultratex
    return ultratex


def cu_tensor(lengths):
    return torch.tensor(o.prefix(lengths), dtype=torch.int32, device="cuda")


def inputs(n, C, dtype, seed=0, shift=0.5):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(n, C, generator=g) * 1.5 + shift * (1 + torch.randn(C, generator=g))).to(dtype).cuda()
    dy = torch.randn(n, C, generator=g).to(dtype).cuda()
    gamma = (1 + 0.2 * torch.randn(C, generator=g)).cuda()
    beta = (0.3 * torch.randn(C, generator=g)).cuda()
    return x, dy, gamma, beta


def close(got, ref, bound, what):
    got = to_np(got)
    assert np.isfinite(got).all(), what
    err = np.abs(got - ref)
    assert (err <= bound).all(), (what, float((err / (bound + 1e-30)).max()))


def check(u, x, dy, gamma, beta, groups, lengths, act, eps=1e-5, one_segment=False, backward=True):
    cu = None if one_segment else cu_tensor(lengths)
    status = u.status_word()
    y, mean, rstd = u.ut_group_norm_fwd(x, gamma, beta, groups, eps=eps, act=act, cu=cu, status=status)
    u.check_status(status)
    C = x.shape[1]
    hx, hdy = to_np(x), to_np(dy)
    hg = to_np(gamma) if gamma is not None else np.ones(C)
    hb = to_np(beta) if beta is not None else np.zeros(C)
    c = o.prefix(lengths)
    ry, rm, rr = o.group_norm_fwd(hx, hg, hb, groups, eps, act, c)
    seg = np.repeat(np.arange(len(lengths)), lengths)
    big = np.array([np.abs(hx[c[s]:c[s + 1]]).max() if c[s] < c[s + 1] else 0.0 for s in range(len(lengths))])
    close(mean, rm, (E * big)[:, None], "mean")
    # a variance of M values around a mean that is off by e is off by e^2
    close(rstd, rr, E * rr * (1 + (big[:, None] * rr) * 2.0 ** -7), "rstd")
    rs, mu = np.repeat(rr, C // groups, 1)[seg], np.repeat(rm, C // groups, 1)[seg]
    xh_mag = (np.abs(hx) + np.abs(mu)) * rs
    close(y, ry, ROUND[x.dtype] * np.abs(ry) + E * (xh_mag * np.abs(hg) + np.abs(hb) + 1e-6), "y")
    if not backward:
        return y, mean, rstd
    dx, dgamma, dbeta = u.ut_group_norm_bwd(x, dy, gamma, beta, mean, rstd, groups, act=act, cu=cu, status=status)
    u.check_status(status)
    r = o.group_norm_bwd(hx, hdy, hg, hb, groups, eps, act, c)
    k = 4 * (1 + (xh_mag.max() if xh_mag.size else 0) / 8)  # act' and xh move with the error of xh
    close(dx, r["dx"], ROUND[x.dtype] * np.abs(r["dx"]) + k * E * (r["dx_abs"] + 1e-6), "dx")
    close(dgamma, r["dgamma"], k * E * (r["dgamma_abs"] + 1e-6), "dgamma")
    close(dbeta, r["dbeta"], k * E * (r["dbeta_abs"] + 1e-6), "dbeta")
    return y, mean, rstd, dx, dgamma, dbeta


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("act", [0, 1])
@pytest.mark.parametrize("lengths", [[1], [2], [257], [1, 0, 33, 700, 5], [0, 0], [4099]])
@pytest.mark.parametrize("channels,groups", [(8, 1), (40, 4), (320, 32), (64, 64)])
def test_lengths_and_groups(u, lengths, channels, groups, act, dtype):
    n = sum(lengths)
    check(u, *inputs(n, channels, dtype, seed=n + channels), groups, lengths, act, one_segment=len(lengths) == 1)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("channels,groups", [(8192, 32), (2056, 8), (1000, 5), (128, 1), (640, 32), (4104, 3)])
def test_wide_rows(u, channels, groups, dtype):
    """Several column chunks per row, groups across 16-byte columns and across chunks."""
    check(u, *inputs(150, channels, dtype, seed=channels), groups, [100, 50], 1)


@pytest.mark.parametrize("lengths", [[60000], [20000, 1, 45000]])
def test_many_rows(u, lengths):
    n = sum(lengths)
    check(u, *inputs(n, 64, torch.bfloat16, seed=3), 8, lengths, 1, one_segment=len(lengths) == 1)


@pytest.mark.parametrize("lengths", [[5000], [17, 3000]])
def test_mean_far_from_zero(u, lengths):
    """Values around 1000 with a spread near 1: a sum of squares would have lost the variance."""
    n = sum(lengths)
    x, dy, gamma, beta = inputs(n, 32, torch.float32, seed=4)
    check(u, x + 1000, dy, gamma, beta, 4, lengths, 0)
    x[0] = -30000.0  # and a first row that is like no other
    check(u, x, dy, gamma, beta, 4, lengths, 1, backward=False)


def test_constant_rows_and_no_affine(u):
    x, dy, _, _ = inputs(300, 64, torch.float32, seed=5)
    check(u, x, dy, None, None, 8, [100, 200], 1)
    x[:] = 2.5
    y, mean, rstd = u.ut_group_norm_fwd(x, None, None, 8, act=0)
    assert torch.all(y == 0) and torch.all(mean == 2.5)
    assert np.allclose(to_np(rstd), 1e5 ** 0.5, rtol=1e-6)


def test_spoilt_segment_stays_alone(u):
    x, dy, gamma, beta = inputs(400, 64, torch.bfloat16, seed=6)
    cu = cu_tensor([150, 100, 150])
    a = u.ut_group_norm_fwd(x, gamma, beta, 8, cu=cu)
    g = u.ut_group_norm_bwd(x, dy, gamma, beta, a[1], a[2], 8, cu=cu)
    x2, dy2 = x.clone(), dy.clone()
    x2[160, 3], dy2[170] = float("nan"), float("inf")
    b = u.ut_group_norm_fwd(x2, gamma, beta, 8, cu=cu)
    g2 = u.ut_group_norm_bwd(x2, dy2, gamma, beta, b[1], b[2], 8, cu=cu)
    rows = list(range(150)) + list(range(250, 400))
    assert torch.equal(a[0][rows], b[0][rows]) and torch.equal(g[0][rows], g2[0][rows])
    assert torch.isnan(b[1][1, 0]) and torch.equal(a[1][1, 1:], b[1][1, 1:])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_strides_streams_and_repeats(u, dtype):
    """Padded rows at bases that are only 16-byte aligned, outputs inside larger buffers, another stream: same bits."""
    e = 16 // torch.empty(0, dtype=dtype).element_size()
    x, dy, gamma, beta = inputs(700, 80, dtype, seed=7)
    cu = cu_tensor([300, 400])
    want = u.ut_group_norm_fwd(x, gamma, beta, 10, cu=cu)
    wantg = u.ut_group_norm_bwd(x, dy, gamma, beta, *want[1:], 10, cu=cu)

    def framed(src=None):
        b = torch.full((702, 80 + 2 * e), 7.0, dtype=dtype, device="cuda")
        v = b[1:-1, e:-e]
        if src is not None:
            v.copy_(src)
        return b, v

    (_, x2), (_, dy2), (by, y), (bd, dx) = framed(x), framed(dy), framed(), framed()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = u.ut_group_norm_fwd(x2, gamma, beta, 10, cu=cu, y=y)
        gotg = u.ut_group_norm_bwd(x2, dy2, gamma, beta, *got[1:], 10, cu=cu, dx=dx)
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip((*want, *wantg), (*got, *gotg)):
        assert torch.equal(a, b)
    for b in (by, bd):
        frame = b.clone()
        frame[1:-1, e:-e] = 7.0
        assert torch.equal(frame, torch.full_like(b, 7.0))


def test_gradient_matches_differences(u):
    x, dy, gamma, beta = inputs(120, 40, torch.float32, seed=8)
    lengths = [50, 70]
    y, mean, rstd = u.ut_group_norm_fwd(x, gamma, beta, 4, cu=cu_tensor(lengths))
    grads = u.ut_group_norm_bwd(x, dy, gamma, beta, mean, rstd, 4, cu=cu_tensor(lengths))
    z, hdy = [to_np(t) for t in (x, gamma, beta)], to_np(dy)
    g = np.random.Generator(np.random.PCG64(2))
    for i in range(3):
        d = g.standard_normal(z[i].shape)
        f = [o.group_norm_fwd(*[t + s * 1e-5 * d if j == i else t for j, t in enumerate(z)], 4, 1e-5, 1,
                              o.prefix(lengths))[0] for s in (1, -1)]
        want = ((f[0] - f[1]) * hdy).sum() / 2e-5
        terms = np.abs(to_np(grads[i]) * d).sum()
        assert abs((to_np(grads[i]) * d).sum() - want) <= 2.0 ** -15 * terms + 1e-6, i


@pytest.mark.parametrize("cu", [[0, 40, 30, 70], [0, 20, 40, 90], [5, 20, 40, 70], [0, -4, 1 << 30, 70]])
def test_wrong_prefix_is_reported(u, cu):
    x, dy, gamma, beta = inputs(70, 64, torch.bfloat16)
    bad = torch.tensor(cu, dtype=torch.int32, device="cuda")
    status = u.status_word()
    _, mean, rstd = u.ut_group_norm_fwd(x, gamma, beta, 8, cu=bad, status=status)
    with pytest.raises(u.UtError, match="invalid argument"):
        u.check_status(status)
    status = u.status_word()
    u.ut_group_norm_bwd(x, dy, gamma, beta, mean, rstd, 8, cu=bad, status=status)
    with pytest.raises(u.UtError, match="invalid argument"):
        u.check_status(status)
    check(u, x, dy, gamma, beta, 8, [70], 1, one_segment=True)


def test_rows_past_32_bit_offsets(u):
    n, C = (1 << 31) // 1024 + 500, 1024
    x = torch.zeros(n, C, dtype=torch.bfloat16, device="cuda")
    tail, _, gamma, beta = inputs(700, C, torch.bfloat16, seed=9)
    x[-700:] = tail
    cu = torch.tensor([0, n - 700, n], dtype=torch.int32, device="cuda")
    y, mean, rstd = u.ut_group_norm_fwd(x, gamma, beta, 32, cu=cu)
    want, wm, wr = u.ut_group_norm_fwd(tail, gamma, beta, 32)
    ref, _, _ = o.group_norm_fwd(to_np(tail), to_np(gamma), to_np(beta), 32, 1e-5, 1, o.prefix([700]))
    close(y[-700:], ref, 2.0 ** -8 * np.abs(ref) + 64 * E, "y")
    assert torch.all(mean[0] == 0) and torch.allclose(mean[1], wm[0], atol=1e-6)
    assert torch.equal(y[0], y[n - 701])


def test_refusals(u):
    x, dy, gamma, beta = inputs(20, 64, torch.bfloat16)
    with pytest.raises(ValueError, match="gamma"):
        u.ut_group_norm_fwd(x, gamma.bfloat16(), beta, 8)
    with pytest.raises(ValueError, match="int32"):
        u.ut_group_norm_fwd(x, gamma, beta, 8, cu=cu_tensor([20]).long())
    with pytest.raises(ValueError, match="contiguous within"):
        u.ut_group_norm_fwd(x.t().contiguous().t(), gamma, beta, 8)
    with pytest.raises(ValueError, match="share one device"):
        u.ut_group_norm_fwd(x, gamma.cpu(), beta, 8)
    with pytest.raises(TypeError):
        u.ut_group_norm_fwd(x.half(), gamma, beta, 8)
    for groups, eps, act in ((7, 1e-5, 1), (8, 0.0, 1), (8, float("nan"), 1), (8, 1e-5, 2)):
        with pytest.raises(u.UtError, match="invalid argument"):
            u.ut_group_norm_fwd(x, gamma, beta, groups, eps=eps, act=act)
    with pytest.raises(u.UtError, match="invalid argument"):
        u.ut_group_norm_fwd(x[:, 4:60], gamma[4:60].contiguous(), beta[4:60].contiguous(), 8)  # base 8-byte aligned
    with pytest.raises(u.UtError, match="unsupported"):
        u.ut_group_norm_fwd(x.repeat(1, 200), None, None, 8)
    y, mean, rstd = u.ut_group_norm_fwd(x, gamma, beta, 8)
    with pytest.raises(u.UtError, match="invalid argument"):
        u.ut_group_norm_bwd(x, dy, gamma, beta, mean, rstd, 8, ws=torch.empty(16, dtype=torch.uint8, device="cuda"))

"""Group norm on rows of several slabs of columns, with enough rows that every block has many chunks of each: against
the float64 oracle with the tolerances of test_gpu_gnorm (no thread sums more rows there than in its longest case), and
inside frames that have to stay untouched."""
import pytest
import torch

from test_gpu_gnorm import check, cu_tensor, inputs, u  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("channels,groups", [(1536, 32), (2048, 32), (2560, 5), (3848, 1), (4096, 32), (8192, 64)])
def test_many_rows_of_several_slabs(u, channels, groups, dtype):  # noqa: F811
    lengths = [1201, 0, 1, 1806]
    n = sum(lengths)
    x, dy, gamma, beta = inputs(n, channels, dtype, seed=channels)
    want = check(u, x, dy, gamma, beta, groups, lengths, 1)
    e = 16 // x.element_size()
    frames = [torch.full((n + 128, channels + 2 * e), 7.0, dtype=dtype, device="cuda") for _ in range(2)]
    y, dx = (f[64:-64, e:-e] for f in frames)
    cu = cu_tensor(lengths)
    got = u.ut_group_norm_fwd(x, gamma, beta, groups, cu=cu, y=y)
    got += u.ut_group_norm_bwd(x, dy, gamma, beta, *got[1:], groups, cu=cu, dx=dx)
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    for f in frames:
        f[64:-64, e:-e] = 7.0
        assert torch.equal(f, torch.full_like(f, 7.0))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("channels,groups", [(8192, 4096), (8192, 2048), (6144, 6144), (7680, 3840)])
def test_limits_of_channels_and_groups(u, channels, groups, dtype):  # noqa: F811
    """The most channels and groups that are accepted, forward and backward; several chunks a block."""
    lengths = [900, 700]
    check(u, *inputs(sum(lengths), channels, dtype, seed=groups), groups, lengths, 1)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_wrong_prefixes_cost_no_waits(u, dtype):  # noqa: F811
    """Prefixes out of order over rows of many chunks: reported as what they are, and no wait runs out on their account."""
    n, channels = 60000, 320
    x, dy, gamma, beta = inputs(n, channels, dtype, seed=2)
    for cu in ([0, 50000, 20000, 60000], [30000, 10, 60000, 0, 60000], [0, 59000, 300, 20, 60000], [60000, 0]):
        bad = torch.tensor(cu, dtype=torch.int32, device="cuda")
        status = u.status_word()
        start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        start.record()
        _, mean, rstd = u.ut_group_norm_fwd(x, gamma, beta, 32, cu=bad, status=status)
        u.ut_group_norm_bwd(x, dy, gamma, beta, mean, rstd, 32, cu=bad, status=status)
        end.record()
        end.synchronize()
        assert int(status.item()) == u.UT_ERR_INVALID_ARG
        assert start.elapsed_time(end) < 500.0  # ms; the limit of one wait is 2,000
    check(u, x, dy, gamma, beta, 32, [n], 1, one_segment=True)


def test_more_statistics_than_32_bits_count(u):  # noqa: F811
    """2^31 and more pairs of segment and group, all but the last segment empty."""
    B, groups, n, eps = (1 << 25) + 3, 64, 10, 1e-5
    x, _, gamma, beta = inputs(n, groups, torch.bfloat16, seed=1)
    cu = torch.zeros(B + 1, dtype=torch.int32, device="cuda")
    cu[-1] = n
    mean, rstd = (torch.full((B, groups), float("nan"), device="cuda") for _ in range(2))
    status = u.status_word()
    y, _, _ = u.ut_group_norm_fwd(x, gamma, beta, groups, eps=eps, cu=cu, mean=mean, rstd=rstd, status=status)
    u.check_status(status)
    want = u.ut_group_norm_fwd(x, gamma, beta, groups, eps=eps)
    assert torch.equal(y, want[0]) and torch.equal(mean[-1:], want[1]) and torch.equal(rstd[-1:], want[2])
    assert int(torch.count_nonzero(mean[:-1])) == 0
    lo, hi = torch.aminmax(rstd[:-1])
    assert lo == hi and abs(lo.item() - eps ** -0.5) <= 2.0 ** -22 * eps ** -0.5

"""Cross attention with values that are not finite: what they spoil shows, what they must not reach keeps its bits."""
import pytest
import torch

from test_gpu_xattn import cu_tensor, inputs, u  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lk", [[77, 20], [128, 40], [300, 77]])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_spoilt_query_row_shows_in_its_gradient_alone(u, value, lk, d, dtype):  # noqa: F811
    """One head of one query row: its O, LSE and dQ are NaN (an infinity gives scores of both signs); other heads and
    rows keep their bits.  Segments of one key block and of several, whole and not, with masked keys and without."""
    lq, heads = [40, 150], 4
    q, k, v, dout = inputs(lq, lk, heads, 2, d, dtype, seed=d)
    mask = (torch.rand(sum(lk), generator=torch.Generator().manual_seed(3)) < 0.7).to(torch.uint8).cuda()
    rows = [7, 170]
    for m in (None, mask):
        how = dict(cu_q=cu_tensor(lq), cu_k=cu_tensor(lk), key_mask=m)
        clean = u.ut_xattn_fwd(q, k, v, **how)
        dq = u.ut_xattn_bwd(q, k, v, *clean, dout, **how)[0]
        q2 = q.clone()
        for r in rows:
            q2[r, 1, 5] = value
        out = u.ut_xattn_fwd(q2, k, v, **how)
        dq2 = u.ut_xattn_bwd(q2, k, v, *out, dout, **how)[0]
        for r in rows:
            assert torch.isnan(out[0][r, 1]).all() and torch.isnan(out[1][1, r]) and torch.isnan(dq2[r, 1]).all()
            for t, c in ((out[0], clean[0]), (dq2, dq)):
                t[r, 1] = c[r, 1]
            out[1][1, r] = clean[1][1, r]
        assert torch.equal(out[0], clean[0]) and torch.equal(out[1], clean[1]) and torch.equal(dq2, dq)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("lq,lk", [([40, 150], [77, 20]), ([300, 9], [300, 129])])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_masked_keys_have_zero_gradients_beside_spoilt_rows(u, value, lq, lk, dtype):  # noqa: F811
    """Rows of Q and dO that are not finite make the gradients of their segment's keys so, not of masked ones; and a
    segment whose keys are all masked has no gradient at all."""
    q, k, v, dout = inputs(lq + [6], lk + [5], 4, 2, 64, dtype, seed=len(lk) + lk[0])
    mask = (torch.rand(sum(lk) + 5, generator=torch.Generator().manual_seed(4)) < 0.5).to(torch.uint8).cuda()
    mask[-5:] = 0
    q[3], dout[5], dout[-2], q[-1] = value, value, value, value
    how = dict(cu_q=cu_tensor(lq + [6]), cu_k=cu_tensor(lk + [5]), key_mask=mask)
    out, lse = u.ut_xattn_fwd(q, k, v, **how)
    dq, dk, dv = u.ut_xattn_bwd(q, k, v, out, lse, dout, **how)
    off = mask == 0
    assert not dk[off].any() and not dv[off].any() and not dq[-6:].any() and not out[-6:].any()
    assert torch.isneginf(lse[:, -6:]).all()
    mine = (mask[:lk[0]] != 0).nonzero()[:, 0]
    assert not torch.isfinite(dv[mine]).any() and torch.isfinite(dv[lk[0]:]).all() and torch.isfinite(dk[lk[0]:]).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("lq,lk", [([200], [300]), ([1], [9000])])
@pytest.mark.parametrize("size", [-2.0 ** 10, 2.0 ** 10, -2.0 ** 14, 2.0 ** 14])
def test_large_scores(u, size, lq, lk, dtype):  # noqa: F811
    """Scores up to 2^28 of either sign.  Each is exact in fp32 and the largest is more than 4,000 above the next, so that
    it has all the weight; blocks before its own hold lower ones, or masked keys only.

    Tolerance, derived: in bf16 the exponent of the largest is its own rounding in base 2 (up to 2^4), so P = 2^x is
    rounded for its product and the sum is not, 2^-8 each for P and O; in fp32 it is 0, and P = 1.  LSE: three roundings
    of 2^-24."""
    n, d, best = lk[0], 64, lk[0] - 40
    q = torch.zeros(lq[0], 2, d, dtype=dtype, device="cuda")
    k = torch.zeros(n, 2, d, dtype=dtype, device="cuda")
    v = inputs(lq, lk, 2, 2, d, dtype, seed=1)[2]
    rank = torch.randperm(n, generator=torch.Generator().manual_seed(2)) % 127  # of sizes that bf16 holds
    rank[best] = 127
    at = (128 + rank if size > 0 else 256 - rank) / 128
    q[..., 0], k[..., 0] = size, (at * abs(size)).to(dtype).cuda()[:, None]
    mask = torch.ones(n, dtype=torch.uint8, device="cuda")
    mask[:140] = 0
    want = float(at[best]) * size * abs(size) * 0.5
    for m in (None, mask):
        out, lse = u.ut_xattn_fwd(q, k, v, key_mask=m, softmax_scale=0.5)
        e = 2.0 ** -7 if dtype == torch.bfloat16 else 0.0
        assert torch.all((out - v[best]).abs().float() <= e * v[best].abs().float())
        assert torch.all((lse - want).abs() <= 2.0 ** -22 * abs(want))

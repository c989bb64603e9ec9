"""Cross attention to an encoder's states against the float64 oracle.

Tolerances (per element, derived, not fitted).  bf16: P (forward, dV) or dS (dQ, dK) is rounded once before its
product and the result once after it, each by at most 2^-8 of a term or of the result; D = dO . O takes O as the
forward rounded it.  So |O err| <= u (|O| + sum p |v|) with u = 2^-8, and alike for the gradients with their terms'
magnitudes plus the error of D; fp32 accumulation, the exponential and the logarithm add less than 1/8 of u.
fp32: S = q . k has d products, whose rounding (2^-24 each, growing as their root) reaches exp(S) times |S|'s scale
of about 8: u = 2^-16 leaves a factor of about 4.  LSE: that error of S alone, 2^-16 for both types."""
import numpy as np
import pytest
import torch

import oracle.conditioning_oracle as o
from gpu_util import need_gpu, to_np

pytestmark = pytest.mark.gpu

U = {torch.bfloat16: 2.0 ** -8 * 1.125, torch.float32: 2.0 ** -16}


@pytest.fixture(scope="module")
def u():
    need_gpu()
    from paper_2609_23169_gb300 import ultratex
    return ultratex


def cu_tensor(lengths):
    return torch.tensor(o.prefix(lengths), dtype=torch.int32, device="cuda")


def inputs(lq, lk, H, Hk, d, dtype, seed=0, fused=False, pad=0):
    g = torch.Generator().manual_seed(seed)
    nq, nk = sum(lq), sum(lk)

    def rows(n, heads, scale=1.0):
        x = (torch.randn(n, heads * d + pad, generator=g) * scale).to(dtype).cuda()
        return x[:, :heads * d].unflatten(1, (heads, d))

    q, dout = rows(nq, H, 1.3), rows(nq, H)
    if fused:
        kv = rows(nk, 2 * Hk).unflatten(1, (2, Hk))
        k, v = kv[:, 0], kv[:, 1]
    else:
        k, v = rows(nk, Hk), rows(nk, Hk)
    return q, k, v, dout


def close(got, ref, bound, what):
    got = to_np(got)
    assert np.isfinite(got).all(), what
    bad = np.abs(got - ref) > bound + 1e-30
    assert not bad.any(), (what, int(bad.sum()), float((np.abs(got - ref) / (bound + 1e-30)).max()))


def check(u, q, k, v, dout, lq, lk, mask=None, scale=None, one_segment=False, backward=True):
    how = {} if one_segment else {"cu_q": cu_tensor(lq), "cu_k": cu_tensor(lk)}
    status = u.status_word()
    how.update(softmax_scale=scale, key_mask=mask, status=status)
    out, lse = u.ut_xattn_fwd(q, k, v, **how)
    u.check_status(status)
    cq, ck = o.prefix(lq), o.prefix(lk)
    m = None if mask is None else mask.cpu().numpy()
    hq, hk, hv, hd = (to_np(t) for t in (q, k, v, dout))
    ref, ref_lse, oabs = o.xattn_fwd(hq, hk, hv, cq, ck, m, scale)
    e = U[q.dtype]
    close(out, ref, e * (np.abs(ref) + oabs), "O")
    seen = np.isfinite(ref_lse)
    got_lse = to_np(lse)
    assert np.all(np.isneginf(got_lse[~seen]))
    assert not to_np(out).transpose(1, 0, 2)[~seen].any()
    assert np.all(np.abs(got_lse[seen] - ref_lse[seen]) <= 2.0 ** -16 * (1 + np.abs(ref_lse[seen])))
    if not backward:
        return out, lse
    grads = u.ut_xattn_bwd(q, k, v, out, lse, dout, **how)
    u.check_status(status)
    r = o.xattn_bwd(hq, hk, hv, hd, cq, ck, m, scale, do_err=e * (np.abs(ref) + oabs))
    for name, g in zip(("dq", "dk", "dv"), grads):
        close(g, r[name], e * (np.abs(r[name]) + r[name + "_abs"]) + r.get(name + "_d", 0.0), name)
    if m is not None:
        assert not to_np(grads[1])[m == 0].any() and not to_np(grads[2])[m == 0].any()
    return out, lse, grads


LENGTHS = [
    ([1], [1]), ([1], [77]), ([3], [128]), ([130], [129]), ([257], [64]), ([64, 1, 0, 129, 7], [77, 0, 300, 1, 128]),
    ([1, 1, 1, 1], [513, 31, 2, 260]), ([0], [5]), ([300], [0]), ([5, 2], [700, 1000]),
]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("heads,kv_heads,d", [(2, 2, 64), (3, 1, 128), (8, 2, 64)])
@pytest.mark.parametrize("lq,lk", LENGTHS)
def test_lengths(u, lq, lk, heads, kv_heads, d, dtype):
    x = inputs(lq, lk, heads, kv_heads, d, dtype, seed=len(lq) + heads)
    check(u, *x, lq, lk, one_segment=len(lq) == 1)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (5, 5), (24, 8), (64, 1), (7, 1), (12, 4)])
def test_head_groups(u, heads, kv_heads, dtype):
    lq, lk = [40, 3, 90], [50, 130, 9]
    check(u, *inputs(lq, lk, heads, kv_heads, 64, dtype, seed=heads), lq, lk)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kind", ["random", "none_left", "first_blocks", "only_last", "one_segment_empty"])
def test_masks(u, kind, dtype):
    lq, lk = [70, 20, 130], [300, 40, 129]
    x = inputs(lq, lk, 4, 2, 64, dtype, seed=5)
    n = sum(lk)
    g = torch.Generator().manual_seed(1)
    mask = (torch.rand(n, generator=g) < 0.5).to(torch.uint8)
    if kind == "none_left":
        mask[:] = 0
    elif kind == "first_blocks":
        mask[:260] = 0
    elif kind == "only_last":
        mask[:] = 0
        mask[[299, 339, 468]] = 7
    elif kind == "one_segment_empty":
        mask[300:340] = 0
    check(u, *x, lq, lk, mask=mask.cuda())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("few", [False, True])
def test_masked_rows_may_hold_anything(u, dtype, few):
    """NaN and infinities in masked keys and values, and in the rows of another segment, reach no result."""
    lq, lk = ([1, 2, 1] if few else [70, 20, 130]), [700, 40, 529]
    q, k, v, dout = inputs(lq, lk, 4, 2, 64, dtype, seed=6)
    mask = (torch.rand(sum(lk), generator=torch.Generator().manual_seed(2)) < 0.6).to(torch.uint8).cuda()
    how = dict(cu_q=cu_tensor(lq), cu_k=cu_tensor(lk), key_mask=mask)
    mask[700:740] = 1
    clean = u.ut_xattn_fwd(q, k, v, **how)
    grads = u.ut_xattn_bwd(q, k, v, *clean, dout, **how)
    k2, v2 = k.clone(), v.clone()
    off = mask == 0
    k2[off], v2[off] = float("nan"), float("inf")
    k2[700:740], v2[700:740] = float("nan"), float("-inf")   # the second segment is spoilt
    q2, dout2 = q.clone(), dout.clone()
    a, b = lq[0], lq[0] + lq[1]
    q2[a:b], dout2[a:b] = float("inf"), float("nan")
    spoilt = u.ut_xattn_fwd(q2, k2, v2, **how)
    grads2 = u.ut_xattn_bwd(q2, k2, v2, *spoilt, dout2, **how)
    rows = [i for i in range(sum(lq)) if not a <= i < b]
    keys = [i for i in range(sum(lk)) if not 700 <= i < 740]
    assert torch.equal(clean[0][rows], spoilt[0][rows]) and torch.equal(clean[1][:, rows], spoilt[1][:, rows])
    assert torch.equal(grads[0][rows], grads2[0][rows])
    for x, y in zip(grads[1:], grads2[1:]):
        assert torch.equal(x[keys], y[keys])
    assert not torch.isfinite(spoilt[0][a:b].float()).any()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("lq,lk", [([1], [5000]), ([3, 1], [2100, 999]), ([24], [1031])])
def test_few_queries_over_long_states(u, lq, lk, dtype):
    """The forms that split the keys: serving of single queries, with masks that leave whole splits empty."""
    x = inputs(lq, lk, 3, 3, 128, dtype, seed=7, fused=True)
    check(u, *x, lq, lk)
    mask = torch.zeros(sum(lk), dtype=torch.uint8)
    mask[lk[0] - 2:lk[0]] = 1
    check(u, *x, lq, lk, mask=mask.cuda(), backward=False)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_strides_and_alignment(u, dtype):
    """K and V as slices of one projection, padded rows, bases that are only 16-byte aligned, outputs inside larger
    buffers whose other values stay untouched, and a mask at an odd address."""
    lq, lk = [45, 100], [90, 33]
    e = 16 // torch.empty(0, dtype=dtype).element_size()
    q, k, v, dout = inputs(lq, lk, 6, 3, 64, dtype, seed=8, fused=True, pad=3 * e)
    base = torch.zeros(145 * 400 + e, dtype=dtype, device="cuda")
    q2 = base[e:e + 145 * 400].view(145, 400)[:, :384].unflatten(1, (6, 64))
    q2.copy_(q)
    mask = torch.ones(sum(lk) + 1, dtype=torch.uint8, device="cuda")[1:]
    mask[10:20] = 0
    how = dict(cu_q=cu_tensor(lq), cu_k=cu_tensor(lk), key_mask=mask)

    def framed(n, width):
        b = torch.full((n + 2, width + 2 * e), 7.0, dtype=dtype, device="cuda")
        return b, b[1:-1, e:e + width]

    bo, oo = framed(145, 384)
    out, lse = u.ut_xattn_fwd(q2, k, v, o=oo.unflatten(1, (6, 64)), **how)
    want, want_lse = u.ut_xattn_fwd(q.contiguous(), k.contiguous(), v.contiguous(), **how)
    assert torch.equal(out, want) and torch.equal(lse, want_lse)
    bq, dq = framed(145, 384)
    bkv, dkv = framed(123, 2 * 192)
    dkv = dkv.unflatten(1, (2, 3, 64))
    u.ut_xattn_bwd(q2, k, v, out, lse, dout, dq=dq.unflatten(1, (6, 64)), dk=dkv[:, 0], dv=dkv[:, 1], **how)
    wq, wk, wv = u.ut_xattn_bwd(q.contiguous(), k.contiguous(), v.contiguous(), want, lse, dout.contiguous(), **how)
    assert torch.equal(dq, wq.flatten(1)) and torch.equal(dkv[:, 0], wk) and torch.equal(dkv[:, 1], wv)
    for b in (bo, bq, bkv):
        frame = b.clone()
        frame[1:-1, e:-e] = 7.0
        assert torch.equal(frame, torch.full_like(b, 7.0))


def test_scale_and_large_scores(u):
    """Scores up to several hundred: the running maximum keeps every exponential finite."""
    lq, lk = [33], [400]
    q, k, v, dout = inputs(lq, lk, 2, 2, 64, torch.float32, seed=9)
    out, lse = u.ut_xattn_fwd(q * 8, k, v, softmax_scale=1.0)
    ref, ref_lse, _ = o.xattn_fwd(to_np(q * 8), to_np(k), to_np(v), o.prefix(lq), o.prefix(lk), None, 1.0)
    assert np.abs(ref_lse).max() > 150
    assert np.abs(to_np(lse) - ref_lse).max() <= 2.0 ** -16 * np.abs(ref_lse).max()
    for dt in (torch.bfloat16, torch.float32):
        x = inputs(lq, lk, 2, 2, 64, dt, seed=10)
        check(u, *x, lq, lk, scale=0.5, one_segment=True)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_same_bits_on_every_run_and_stream(u, dtype):
    """The forward, dK and dV repeat to the bit, on another stream too (ordered after the inputs by an event)."""
    lq, lk = [200, 31], [300, 77]
    x = inputs(lq, lk, 4, 4, 64, dtype, seed=11)
    how = dict(cu_q=cu_tensor(lq), cu_k=cu_tensor(lk))
    first = u.ut_xattn_fwd(*x[:3], **how)
    g1 = u.ut_xattn_bwd(*x[:3], *first, x[3], **how)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = u.ut_xattn_fwd(*x[:3], **how)
        g2 = u.ut_xattn_bwd(*x[:3], *again, x[3], **how)
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip((*first, g1[1], g1[2]), (*again, g2[1], g2[2])):
        assert torch.equal(a, b)


def test_gradient_matches_differences(u):
    """fp32 gradients against central differences of the float64 forward along random directions."""
    lq, lk = [9, 20], [70, 5]
    x = inputs(lq, lk, 4, 2, 64, torch.float32, seed=12)
    how = dict(cu_q=cu_tensor(lq), cu_k=cu_tensor(lk))
    out, lse = u.ut_xattn_fwd(*x[:3], **how)
    grads = u.ut_xattn_bwd(*x[:3], out, lse, x[3], **how)
    y, dout = [to_np(t) for t in x[:3]], to_np(x[3])
    g = np.random.Generator(np.random.PCG64(1))
    for i in range(3):
        d = g.standard_normal(y[i].shape)
        f = [o.xattn_fwd(*[t + s * 1e-5 * d if j == i else t for j, t in enumerate(y)], o.prefix(lq), o.prefix(lk))[0]
             for s in (1, -1)]
        want = ((f[0] - f[1]) * dout).sum() / 2e-5
        terms = np.abs(to_np(grads[i]) * d).sum()
        assert abs((to_np(grads[i]) * d).sum() - want) <= 2.0 ** -16 * terms + 1e-6, i


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("cu", [[0, 40, 30, 70], [0, 20, 40, 90], [5, 20, 40, 70], [0, -4, 1 << 30, 70]])
def test_wrong_prefix_is_reported(u, cu, dtype):
    """A prefix out of order or out of range is reported in the status word; nothing outside the tensors is touched."""
    q, k, v, dout = inputs([70], [70], 2, 2, 64, dtype)
    bad = torch.tensor(cu, dtype=torch.int32, device="cuda")
    good = cu_tensor([20, 20, 30])
    for cq, ck in ((bad, good), (good, bad)):
        status = u.status_word()
        out, lse = u.ut_xattn_fwd(q, k, v, cu_q=cq, cu_k=ck, status=status)
        with pytest.raises(u.UtError, match="invalid argument"):
            u.check_status(status)
        status = u.status_word()
        u.ut_xattn_bwd(q, k, v, out, lse, dout, cu_q=cq, cu_k=ck, status=status)
        with pytest.raises(u.UtError, match="invalid argument"):
            u.check_status(status)
    check(u, q, k, v, dout, [70], [70], one_segment=True)


def test_rows_past_32_bit_offsets(u):
    """Encoder rows whose element offsets pass 2^31: only the last rows are kept, so the result is known exactly."""
    nk, H, d = (1 << 31) // 512 + 300, 4, 128
    k = torch.zeros(nk, H, d, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    q = torch.randn(2, H, d, generator=torch.Generator().manual_seed(3)).bfloat16().cuda()
    k[-3:], v[-3:] = torch.randn(2, 3, H, d, generator=torch.Generator().manual_seed(4)).bfloat16().cuda()
    mask = torch.zeros(nk, dtype=torch.uint8, device="cuda")
    mask[-3:] = 1
    out, lse = u.ut_xattn_fwd(q, k, v, key_mask=mask)
    want, want_lse, oabs = o.xattn_fwd(*(to_np(t) for t in (q, k[-3:], v[-3:])), o.prefix([2]), o.prefix([3]))
    close(out, want, U[torch.bfloat16] * (np.abs(want) + oabs), "O")
    assert np.abs(to_np(lse) - want_lse).max() <= 2.0 ** -16 * (1 + np.abs(want_lse).max())


def test_refusals(u):
    q, k, v, dout = inputs([8], [9], 4, 2, 64, torch.bfloat16)
    with pytest.raises(ValueError, match="cu_q"):
        u.ut_xattn_fwd(q, k, v, cu_q=cu_tensor([8]))
    with pytest.raises(ValueError, match="int32"):
        u.ut_xattn_fwd(q, k, v, cu_q=cu_tensor([8]).long(), cu_k=cu_tensor([9]))
    with pytest.raises(ValueError, match="v must be"):
        u.ut_xattn_fwd(q, k, v[:8])
    with pytest.raises(ValueError, match="v must be"):
        u.ut_xattn_fwd(q, k, v.float())
    with pytest.raises(ValueError, match="contiguous within"):
        u.ut_xattn_fwd(q.transpose(0, 1).contiguous().transpose(0, 1), k, v)
    with pytest.raises(ValueError, match="key_mask"):
        u.ut_xattn_fwd(q, k, v, key_mask=torch.ones(8, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError, match="share one device"):
        u.ut_xattn_fwd(q, k, v.cpu())
    with pytest.raises(TypeError):
        u.ut_xattn_fwd(q.half(), k.half(), v.half())
    with pytest.raises(u.UtError, match="invalid argument"):
        u.ut_xattn_fwd(q, k, v, softmax_scale=float("inf"))
    with pytest.raises(u.UtError, match="invalid argument"):
        u.ut_xattn_fwd(q[:, :3].contiguous(), k, v)
    with pytest.raises(u.UtError, match="unsupported"):
        u.ut_xattn_fwd(q[:, :, :32].contiguous(), k[:, :, :32].contiguous(), v[:, :, :32].contiguous())
    out, lse = u.ut_xattn_fwd(q, k, v)
    with pytest.raises(u.UtError, match="invalid argument"):
        u.ut_xattn_bwd(q, k, v, out, lse, dout, ws=torch.empty(64, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError, match="contiguous within"):
        u.ut_xattn_bwd(q, k, v, out, lse, torch.ones((), dtype=q.dtype, device="cuda").expand(q.shape))

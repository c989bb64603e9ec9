"""Windowed attention with visible first keys against the float64 oracle.

Tolerances (per element, derived, not fitted): those of cross attention, whose arithmetic this is.  bf16: P (forward,
dV) or dS (dQ, dK) is rounded at most once before its product and the result once after it, each by at most 2^-8 of a
term or of the result; D = dO . O takes O as the forward rounded it.  So |O err| <= u (|O| + sum p |v|) with u = 2^-8,
and alike for the gradients with their terms' magnitudes plus the error of D; fp32 accumulation, the exponential and
the logarithm add less than 1/8 of u.  fp32: S = q . k has d products, whose rounding (2^-24 each, growing as their
root) reaches exp(S) times |S|'s scale of about 8: u = 2^-16 leaves a factor of about 4.  LSE: that error of S alone,
2^-16 for both types."""
import numpy as np
import pytest
import torch

import oracle.window_oracle as o
from gpu_util import need_gpu, to_np

pytestmark = pytest.mark.gpu

U = {torch.bfloat16: 2.0 ** -8 * 1.125, torch.float32: 2.0 ** -16}
BOTH = pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])


@pytest.fixture(scope="module")
def u():
    need_gpu()
    from paper_2609_23169_gb300 import ultratex
    return ultratex


def prefix(lengths):
    return np.concatenate([[0], np.cumsum(lengths)])


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def inputs(nq, nk, H, Hk, d, dtype, seed=0, fused=False, pad=0):
    g = torch.Generator().manual_seed(seed)

    def rows(n, heads, scale=1.0):
        x = (torch.randn(n, heads * d + pad, generator=g) * scale).to(dtype).cuda()
        return x[:, :heads * d].unflatten(1, (heads, d))

    q, dout = rows(nq, H, 1.3), rows(nq, H)
    if fused:
        kv = rows(nk, 2 * Hk).unflatten(1, (2, Hk))
        return q, kv[:, 0], kv[:, 1], dout
    return q, rows(nk, Hk), rows(nk, Hk), dout


def close(got, ref, bound, what):
    got = to_np(got)
    assert np.isfinite(got).all(), what
    bad = np.abs(got - ref) > bound + 1e-30
    assert not bad.any(), (what, int(bad.sum()), float((np.abs(got - ref) / (bound + 1e-30)).max()))


def check(u, x, lq, lk, win, k_len=None, mask=None, scale=None, backward=True):
    """lk: rows of k and v in each segment (a capacity where there is a k_len)."""
    q, k, v, dout = x
    status = u.status_word()
    how = dict(left=win[0], right=win[1], sinks=win[2], softmax_scale=scale, key_mask=mask, status=status)
    if len(lq) > 1:
        how.update(cu_q=i32(prefix(lq)), cu_k=i32(prefix(lk)))
    if k_len is not None:
        how["k_len"] = i32(k_len)
    out, lse = u.ut_window_attn_fwd(q, k, v, **how)
    u.check_status(status)
    m = None if mask is None else mask.cpu().numpy()
    ref_how = (prefix(lq), prefix(lk), win, k_len, m, scale)
    hq, hk, hv, hd = (to_np(t) for t in x)
    ref, ref_lse, oabs = o.window_fwd(hq, hk, hv, *ref_how)
    e = U[q.dtype]
    close(out, ref, e * (np.abs(ref) + oabs), "O")
    seen, got_lse = np.isfinite(ref_lse), to_np(lse)
    assert np.all(np.isneginf(got_lse[~seen]))
    assert not to_np(out).transpose(1, 0, 2)[~seen].any()
    assert np.all(np.abs(got_lse[seen] - ref_lse[seen]) <= 2.0 ** -16 * (1 + np.abs(ref_lse[seen])))
    if not backward:
        return out, lse
    grads = u.ut_window_attn_bwd(q, k, v, out, lse, dout, **how)
    u.check_status(status)
    r = o.window_bwd(hq, hk, hv, hd, *ref_how, do_err=e * (np.abs(ref) + oabs))
    for name, g in zip(("dq", "dk", "dv"), grads):
        close(g, r[name], e * (np.abs(r[name]) + r[name + "_abs"]) + r.get(name + "_d", 0.0), name)
    # exact zeros where there is no pair of a query and a key
    assert not to_np(grads[0]).transpose(1, 0, 2)[~seen].any()
    unseen = ~r["dv_abs"].any(axis=(1, 2))
    assert not to_np(grads[1])[unseen].any() and not to_np(grads[2])[unseen].any()
    return out, lse, grads


WINDOWS = [(0, 0, 0), (5, 0, 0), (0, 3, 1), (40, 17, 0), (100, 0, 4), (63, 64, 77), (130, 130, 128), (10 ** 9, 0, 0),
           (2 ** 31 + 5, 2 ** 31 + 5, 0), (3, 0, 10 ** 9), (7, 300, 129)]
LENGTHS = [[1], [2], [129], [385], [64, 1, 0, 130, 7], [200, 257, 300]]


@BOTH
@pytest.mark.parametrize("heads,kv_heads,d", [(2, 2, 64), (3, 1, 128)])
@pytest.mark.parametrize("lengths", LENGTHS)
@pytest.mark.parametrize("win", WINDOWS)
def test_windows(u, win, lengths, heads, kv_heads, d, dtype):
    x = inputs(sum(lengths), sum(lengths), heads, kv_heads, d, dtype, seed=len(lengths) + heads)
    check(u, x, lengths, lengths, win)


@BOTH
@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (5, 5), (24, 8), (64, 1), (7, 1), (12, 4)])
def test_head_groups(u, heads, kv_heads, dtype):
    lq, lk = [40, 3, 90], [50, 130, 90]
    check(u, inputs(133, 270, heads, kv_heads, 64, dtype, seed=heads), lq, lk, (20, 2, 5))


@BOTH
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lq,lk", [([5], [3]), ([300], [0]), ([0], [9]), ([200, 4, 0], [70, 4, 33]), ([3, 300], [300, 3])])
def test_more_and_fewer_queries_than_keys(u, lq, lk, d, dtype):
    """Queries before the first key see nothing, or what lies within `right` of them."""
    for win in ((6, 0, 2), (0, 4, 0), (50, 250, 0)):
        check(u, inputs(sum(lq), sum(lk), 4, 2, d, dtype, seed=3), lq, lk, win)


@BOTH
@pytest.mark.parametrize("kind", ["random", "none_left", "first_blocks", "only_last", "one_segment_empty", "sinks_masked"])
def test_masks(u, kind, dtype):
    lk = [300, 40, 329]
    n = sum(lk)
    mask = (torch.rand(n, generator=torch.Generator().manual_seed(1)) < 0.5).to(torch.uint8)
    if kind == "none_left":
        mask[:] = 0
    elif kind == "first_blocks":
        mask[:260] = 0
    elif kind == "only_last":
        mask[:] = 0
        mask[[299, 339, 668]] = 7
    elif kind == "one_segment_empty":
        mask[300:340] = 0
    elif kind == "sinks_masked":
        mask[:9] = mask[300:309] = mask[340:349] = 0
    x = inputs(n, n, 4, 2, 64, dtype, seed=5)
    for win in ((70, 0, 9), (10, 30, 0)):
        check(u, x, lk, lk, win, mask=mask.cuda())


@BOTH
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lq,caps,k_len", [
    ([1], [700], [700]), ([1, 1, 1, 1], [400] * 4, [400, 1, 37, 399]), ([3, 1, 24], [600, 50, 1100], [514, 1, 1031]),
    ([2, 2], [100, 90], [0, 1]), ([13], [5000], [4100]), ([1, 0, 2], [3000, 10, 2000], [2999, 4, 0]),
])
def test_new_tokens_over_caches(u, lq, caps, k_len, d, dtype):
    """Queries at the end of what their caches hold; rows behind it hold NaN.  The forms that split the keys are
    among these."""
    q, k, v, dout = inputs(sum(lq), sum(caps), 6, 2, d, dtype, seed=7)
    at = prefix(caps)
    for s, n in enumerate(k_len):
        k[at[s] + n:at[s + 1]] = float("nan")
        v[at[s] + n:at[s + 1]] = float("nan")
    clean = (q, torch.nan_to_num(k), torch.nan_to_num(v), dout)
    for win in ((100, 0, 4), (3000, 0, 130), (10 ** 6, 0, 0)):
        out, lse, grads = check(u, clean, lq, caps, win, k_len=k_len)
        how = dict(left=win[0], right=win[1], sinks=win[2], k_len=i32(k_len))
        if len(lq) > 1:
            how.update(cu_q=i32(prefix(lq)), cu_k=i32(prefix(caps)))
        out2, lse2 = u.ut_window_attn_fwd(q, k, v, **how)
        assert torch.equal(out, out2) and torch.equal(lse, lse2)
        for a, b in zip(grads, u.ut_window_attn_bwd(q, k, v, out2, lse2, dout, **how)):
            assert torch.equal(a, b)


@BOTH
@pytest.mark.parametrize("n", [1, 3, 40])
def test_rows_that_no_query_sees_may_hold_anything(u, n, dtype):
    """Between the first keys and the window of the last n queries, NaN and infinities reach nothing."""
    nk, win = 900, (100, 0, 70)
    q, k, v, dout = inputs(n, nk, 4, 2, 128, dtype, seed=8)
    out, lse, grads = check(u, (q, k, v, dout), [n], [nk], win)
    gone = slice(win[2], nk - n - win[0])
    k[gone], v[gone] = float("nan"), float("-inf")
    how = dict(left=win[0], sinks=win[2])
    out2, lse2 = u.ut_window_attn_fwd(q, k, v, **how)
    assert torch.equal(out, out2) and torch.equal(lse, lse2)
    for a, b in zip(grads, u.ut_window_attn_bwd(q, k, v, out2, lse2, dout, **how)):
        assert torch.equal(a, b)


@BOTH
def test_masked_and_foreign_rows_may_hold_anything(u, dtype):
    lengths, win = [170, 140, 230], (60, 20, 5)
    n = sum(lengths)
    q, k, v, dout = inputs(n, n, 4, 2, 64, dtype, seed=6)
    mask = (torch.rand(n, generator=torch.Generator().manual_seed(2)) < 0.6).to(torch.uint8).cuda()
    mask[170:310] = 1
    how = dict(left=win[0], right=win[1], sinks=win[2], cu_q=i32(prefix(lengths)), cu_k=i32(prefix(lengths)), key_mask=mask)
    clean = u.ut_window_attn_fwd(q, k, v, **how)
    grads = u.ut_window_attn_bwd(q, k, v, *clean, dout, **how)
    k2, v2, q2, dout2 = k.clone(), v.clone(), q.clone(), dout.clone()
    k2[mask == 0], v2[mask == 0] = float("nan"), float("inf")
    mid = slice(170, 310)   # the second segment is spoilt
    k2[mid], v2[mid], q2[mid], dout2[mid] = float("nan"), float("-inf"), float("inf"), float("nan")
    spoilt = u.ut_window_attn_fwd(q2, k2, v2, **how)
    grads2 = u.ut_window_attn_bwd(q2, k2, v2, *spoilt, dout2, **how)
    rest = torch.ones(n, dtype=torch.bool)
    rest[mid] = False
    assert torch.equal(clean[0][rest], spoilt[0][rest]) and torch.equal(clean[1][:, rest], spoilt[1][:, rest])
    for a, b in zip(grads, grads2):
        assert torch.equal(a[rest], b[rest])
    assert not torch.isfinite(spoilt[0][mid].float()).any()


@BOTH
def test_strides_and_alignment(u, dtype):
    """Slices of one projection, padded rows, bases that are only 16-byte aligned, outputs inside larger buffers whose
    other values stay untouched, and a mask at an odd address."""
    lengths, win = [45, 100], (30, 9, 3)
    e = 16 // torch.empty(0, dtype=dtype).element_size()
    q, k, v, dout = inputs(145, 145, 6, 3, 64, dtype, seed=8, fused=True, pad=3 * e)
    base = torch.zeros(145 * 400 + e, dtype=dtype, device="cuda")
    q2 = base[e:e + 145 * 400].view(145, 400)[:, :384].unflatten(1, (6, 64))
    q2.copy_(q)
    mask = torch.ones(146, dtype=torch.uint8, device="cuda")[1:]
    mask[10:20] = 0
    cu = i32(prefix(lengths))
    how = dict(left=win[0], right=win[1], sinks=win[2], cu_q=cu, cu_k=cu, key_mask=mask)

    def framed(n, width):
        b = torch.full((n + 2, width + 2 * e), 7.0, dtype=dtype, device="cuda")
        return b, b[1:-1, e:e + width]

    bo, oo = framed(145, 384)
    out, lse = u.ut_window_attn_fwd(q2, k, v, o=oo.unflatten(1, (6, 64)), **how)
    want, want_lse = u.ut_window_attn_fwd(q.contiguous(), k.contiguous(), v.contiguous(), **how)
    assert torch.equal(out, want) and torch.equal(lse, want_lse)
    bq, dq = framed(145, 384)
    bkv, dkv = framed(145, 2 * 192)
    dkv = dkv.unflatten(1, (2, 3, 64))
    u.ut_window_attn_bwd(q2, k, v, out, lse, dout, dq=dq.unflatten(1, (6, 64)), dk=dkv[:, 0], dv=dkv[:, 1], **how)
    wq, wk, wv = u.ut_window_attn_bwd(q.contiguous(), k.contiguous(), v.contiguous(), want, lse, dout.contiguous(), **how)
    assert torch.equal(dq, wq.flatten(1)) and torch.equal(dkv[:, 0], wk) and torch.equal(dkv[:, 1], wv)
    for b in (bo, bq, bkv):
        frame = b.clone()
        frame[1:-1, e:-e] = 7.0
        assert torch.equal(frame, torch.full_like(b, 7.0))


@BOTH
def test_scale_and_large_scores(u, dtype):
    x = inputs(333, 333, 2, 2, 64, dtype, seed=10)
    check(u, x, [333], [333], (90, 30, 4), scale=0.5)


@BOTH
@pytest.mark.parametrize("n,win", [(700, (128, 128, 20)), (2, (600, 0, 4))])
def test_same_bits_on_every_run_and_stream_and_in_graphs(u, n, win, dtype):
    """Every output repeats to the bit: again, on another stream, and in two graphs that are replayed side by side, each
    with a workspace of its own."""
    nk = 700
    x = inputs(n, nk, 4, 4, 64, dtype, seed=11)
    how = dict(left=win[0], right=win[1], sinks=win[2])

    def both():
        f = u.ut_window_attn_fwd(*x[:3], **how)
        return (*f, *u.ut_window_attn_bwd(*x[:3], *f, x[3], **how))

    first = both()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = both()
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs = both()
        graphs.append((g, outs, torch.cuda.Stream()))
    for _ in range(3):
        for g, _, s in graphs:
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for other in (again, graphs[0][1], graphs[1][1]):
        for a, b in zip(first, other):
            assert torch.equal(a, b)


def test_gradient_matches_differences(u):
    """fp32 gradients against central differences of the float64 forward along random directions."""
    lengths, win = [9, 70], (15, 3, 2)
    x = inputs(79, 79, 4, 2, 64, torch.float32, seed=12)
    cu = i32(prefix(lengths))
    how = dict(left=win[0], right=win[1], sinks=win[2], cu_q=cu, cu_k=cu)
    out, lse = u.ut_window_attn_fwd(*x[:3], **how)
    grads = u.ut_window_attn_bwd(*x[:3], out, lse, x[3], **how)
    y, dout = [to_np(t) for t in x[:3]], to_np(x[3])
    g = np.random.Generator(np.random.PCG64(1))
    c = prefix(lengths)
    for i in range(3):
        d = g.standard_normal(y[i].shape)
        f = [o.window_fwd(*[t + s * 1e-5 * d if j == i else t for j, t in enumerate(y)], c, c, win)[0] for s in (1, -1)]
        want = ((f[0] - f[1]) * dout).sum() / 2e-5
        terms = np.abs(to_np(grads[i]) * d).sum()
        assert abs((to_np(grads[i]) * d).sum() - want) <= 2.0 ** -16 * terms + 1e-6, i


@BOTH
@pytest.mark.parametrize("what,bad", [("cu", [0, 40, 30, 70]), ("cu", [5, 20, 40, 70]), ("cu", [0, -4, 1 << 30, 70]),
                                      ("k_len", [20, 21, 30]), ("k_len", [-1, 20, 30])])
def test_wrong_lengths_are_reported(u, what, bad, dtype):
    """A prefix out of order or out of range, and a number of keys beyond its segment, are reported in the status word;
    nothing outside the tensors is touched."""
    x = inputs(70, 70, 2, 2, 64, dtype)
    good = i32([0, 20, 40, 70])
    calls = [dict(cu_q=i32(bad), cu_k=good), dict(cu_q=good, cu_k=i32(bad))]
    if what == "k_len":
        calls = [dict(cu_q=good, cu_k=good, k_len=i32(bad))]
    for how in calls:
        status = u.status_word()
        out, lse = u.ut_window_attn_fwd(*x[:3], left=9, sinks=2, status=status, **how)
        with pytest.raises(u.UtError, match="invalid argument"):
            u.check_status(status)
        status = u.status_word()
        u.ut_window_attn_bwd(*x[:3], out, lse, x[3], left=9, sinks=2, status=status, **how)
        with pytest.raises(u.UtError, match="invalid argument"):
            u.check_status(status)
    check(u, x, [70], [70], (9, 0, 2))


def test_rows_past_32_bit_offsets(u):
    """A cache whose element offsets pass 2^31: queries at its end, with first keys at its begin."""
    nk, H, d = (1 << 31) // 512 + 300, 4, 128
    k = torch.zeros(nk, H, d, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    q = torch.randn(2, H, d, generator=torch.Generator().manual_seed(3)).bfloat16().cuda()
    for rows in (slice(0, 4), slice(nk - 203, nk)):
        n = rows.stop - rows.start
        k[rows], v[rows] = torch.randn(2, n, H, d, generator=torch.Generator().manual_seed(n)).bfloat16().cuda()
    out, lse = u.ut_window_attn_fwd(q, k, v, 200, 0, 4)
    keep = torch.cat((torch.arange(4), torch.arange(nk - 203, nk))).cuda()
    # rows between are seen by none; 201 keys and the row's own, then the first four
    ks, vs = to_np(k[keep]), to_np(v[keep])
    want, want_lse, oabs = o.window_fwd(to_np(q), ks, vs, prefix([2]), prefix([207]), (200, 0, 4))
    close(out, want, U[torch.bfloat16] * (np.abs(want) + oabs), "O")
    assert np.abs(to_np(lse) - want_lse).max() <= 2.0 ** -16 * (1 + np.abs(want_lse).max())


def test_as_cross_attention_without_a_window(u):
    """With every key in the window it is cross attention: the same definition, another kernel."""
    x = inputs(130, 130, 4, 2, 64, torch.float32, seed=13)
    a = u.ut_window_attn_fwd(*x[:3], left=130, right=130)
    b = u.ut_xattn_fwd(*x[:3])
    for s, t in zip(a, b):
        assert (s - t).abs().max() <= 2.0 ** -16 * 8


@BOTH
def test_two_calls_at_once(u, dtype):
    """Different problems on two streams at the same time, each with its own workspace."""
    probs = [(inputs(400, 400, 4, 2, 64, dtype, seed=20), (50, 0, 3)), (inputs(3, 3000, 4, 4, 128, dtype, seed=21), (2500, 0, 9))]
    want = [u.ut_window_attn_fwd(*x[:3], *w) for x, w in probs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in probs]
    got = [[], []]
    for _ in range(4):
        for i, (x, w) in enumerate(probs):
            with torch.cuda.stream(streams[i]):
                got[i].append(u.ut_window_attn_fwd(*x[:3], *w))
    torch.cuda.synchronize()
    for i in range(2):
        for o1, l1 in got[i]:
            assert torch.equal(o1, want[i][0]) and torch.equal(l1, want[i][1])

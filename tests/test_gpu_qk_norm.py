"""Norms of queries and keys with the position rotation against the float64 oracle.

Tolerances (per element, derived before the first run).  Forward: the norm and the weight carry a few fp32 roundings
(sum of d squares 2^-20 at worst, half of that in the root, rsqrt 2^-22), the angle is off by 2^-32 turns and by the
fp32 conversion of a part of a turn (2^-24 of at most pi), sine and cosine by 2^-22: together below 2^-19 of the pair's
magnitude, then one rounding to the type, 2^-8 (bf16) or 2^-24 (fp32) of the value.  Backward: two such factors and one
more mean, 2^-18 of the terms' magnitudes.  dw: a lane adds at most 64 tokens' terms in these tests, then 16 lanes, then
at most 54 partial sums: 134 roundings of 2^-24, below 2^-16 of the terms' magnitudes with the terms' own error."""
import numpy as np
import pytest
import torch

import oracle.window_oracle as o
from gpu_util import need_gpu, to_np

pytestmark = pytest.mark.gpu

ROUND = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
BOTH = pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
EPS = 1e-6


@pytest.fixture(scope="module")
def u():
    need_gpu()
    from paper_2609_23169_gb300 import ultratex
    return ultratex


def rope_of(u, kind, d):
    """(binding's rope, oracle's arguments)"""
    if kind == "line":
        return u.rope_config(1, (d, 0, 0), 10000.0), (1, (d, 0, 0), 10000.0, 0)
    axes = (d // 8, (d - d // 8) // 2, (d - d // 8) // 2)
    return u.rope_config(24, axes, 10000.0, 77), (24, axes, 10000.0, 77)


def inputs(n, H, Hk, d, dtype, seed=0, fused=True):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    if fused:
        qkv = (r(n, H + 2 * Hk, d) * 1.5).to(dtype).cuda()
        q, k, v = qkv[:, :H], qkv[:, H:H + Hk], qkv[:, H + Hk:]
    else:
        q, k, v = (r(n, h, d).to(dtype).cuda() for h in (H, Hk, Hk))
    wq, wk = (1 + 0.2 * r(d)).cuda(), (1 + 0.2 * r(d)).cuda()
    return q, k, v, wq, wk, r(n, H, d).to(dtype).cuda(), r(n, Hk, d).to(dtype).cuda()


def close(got, ref, bound, what):
    got = to_np(got)
    assert np.isfinite(got).all(), what
    bad = np.abs(got - ref) > bound + 1e-30
    assert not bad.any(), (what, int(bad.sum()), float((np.abs(got - ref) / (bound + 1e-30)).max()))


def check(u, x, rope, pos, eps=EPS, far=0.0):
    q, k, v, wq, wk, dqo, dko = x
    cfg, args = rope
    ang = o.angles(range(q.shape[0]) if pos is None else pos.tolist(), *args)
    t = ROUND[q.dtype]
    outs = u.ut_qk_norm_rope_fwd(q, k, cfg, wq=wq, wk=wk, eps=eps, pos=pos)
    grads = u.ut_qk_norm_rope_bwd(q, k, cfg, dqo, dko, wq=wq, wk=wk, eps=eps, pos=pos)
    for i, (a, w, dy) in enumerate(((q, wq, dqo), (k, wk, dko))):
        hw = np.ones(q.shape[2]) if w is None else to_np(w)
        ref, size = o.qk_norm_rope(to_np(a), hw, eps, ang)
        close(outs[i], ref, t * np.abs(ref) + (2.0 ** -19 + far) * size, "qk"[i])
        dx, dw, dx_abs, dw_abs = o.qk_norm_rope_bwd(to_np(a), hw, eps, ang, to_np(dy))
        close(grads[i], dx, t * np.abs(dx) + (2.0 ** -18 + far) * dx_abs, "d" + "qk"[i])
        close(grads[2 + i], dw, (2.0 ** -16 + far) * dw_abs, "dw" + "qk"[i])
    return outs, grads


@BOTH
@pytest.mark.parametrize("kind", ["line", "canvas"])
@pytest.mark.parametrize("n,H,Hk,d", [(1, 1, 1, 64), (2, 24, 8, 64), (5, 3, 5, 128), (130, 8, 4, 64), (77, 7, 1, 128),
                                      (1000, 5, 2, 64), (3, 1, 9, 64), (64, 64, 1, 128)])
def test_sizes(u, n, H, Hk, d, kind, dtype):
    x = inputs(n, H, Hk, d, dtype, seed=n + H, fused=n % 2 == 0)
    g = np.random.Generator(np.random.PCG64(n))
    pos = torch.tensor(np.sort(g.integers(-3, 77 + 5 * 576, n)), dtype=torch.int32, device="cuda")
    check(u, x, rope_of(u, kind, d), pos)


@BOTH
def test_default_positions_and_no_weights(u, dtype):
    x = list(inputs(300, 4, 2, 64, dtype, seed=1))
    check(u, x, rope_of(u, "line", 64), None)
    x[3] = x[4] = None
    check(u, x, rope_of(u, "canvas", 64), None, eps=0.5)


@BOTH
def test_far_positions(u, dtype):
    """Positions up to 131,072 cost nothing; at 2^31 - 1 the frequency's 53 bits leave 2^-20 turns (here: 8 radians
    times 2^-20 at most)."""
    x = inputs(6, 4, 2, 64, dtype, seed=2)
    near = torch.tensor([131071, 131072, 100003, 65537, 99991, 120000], dtype=torch.int32, device="cuda")
    check(u, x, rope_of(u, "line", 64), near)
    far = torch.tensor([2 ** 31 - 1, 2 ** 30, 2 ** 31 - 77, 16777217, -2 ** 31, -1], dtype=torch.int32, device="cuda")
    check(u, x, rope_of(u, "line", 64), far, far=8 * 2.0 ** -20)


@BOTH
def test_large_images(u, dtype):
    """A side whose area passes 32 bits: one image holds every position."""
    x = inputs(3, 2, 2, 64, dtype, seed=3)
    args = (70000, (8, 28, 28), 10000.0, 5)
    pos = torch.tensor([5, 2 ** 31 - 1, 70000 * 3 + 11], dtype=torch.int32, device="cuda")
    check(u, x, (u.rope_config(*args), args), pos, far=8 * 2.0 ** -20)


@BOTH
def test_heads_of_zeros_and_of_one_size(u, dtype):
    x = inputs(9, 4, 2, 64, dtype, seed=4)
    x[0][2], x[1][5] = 0, 0
    x[0][3], x[1][4] = 2.0 ** 40, 2.0 ** -40
    check(u, x, rope_of(u, "line", 64), None)


@BOTH
@pytest.mark.parametrize("n", [1, 4, 333])
def test_cache_rows(u, n, dtype):
    """Keys and values go to the given rows; the others stay as they are; negative rows write none."""
    q, k, v, wq, wk, _, _ = inputs(n, 6, 2, 64, dtype, seed=5)
    rope, _ = rope_of(u, "line", 64)
    pos = torch.arange(n, dtype=torch.int32, device="cuda") + 50
    want = u.ut_qk_norm_rope_fwd(q, k, rope, v=v, wq=wq, wk=wk, pos=pos)
    assert torch.equal(want[2], v)
    g = torch.Generator().manual_seed(n)
    rows = torch.randperm(700, generator=g)[:n].int()
    if n > 2:
        rows[1] = -1
    e = 16 // torch.empty(0, dtype=dtype).element_size()
    big = torch.full((700, 2 * 2 * 64 + e), 3.0, dtype=dtype, device="cuda")
    kc, vc = (big[:, i * 128:i * 128 + 128].unflatten(1, (2, 64)) for i in range(2))
    status = u.status_word()
    got = u.ut_qk_norm_rope_fwd(q, k, rope, v=v, wq=wq, wk=wk, pos=pos, rows=rows.cuda(), k_out=kc, v_out=vc, status=status)
    u.check_status(status)
    assert got[1] is kc and got[2] is vc and torch.equal(got[0], want[0])
    ref = torch.full_like(big, 3.0)
    for i in range(n):
        if rows[i] >= 0:
            ref[rows[i], :128], ref[rows[i], 128:256] = want[1][i].flatten(), want[2][i].flatten()
    assert torch.equal(big, ref)


@BOTH
def test_rows_behind_the_cache_are_reported(u, dtype):
    q, k, v, wq, wk, _, _ = inputs(5, 2, 2, 64, dtype, seed=6)
    rope, _ = rope_of(u, "line", 64)
    cache = torch.full((12, 2, 64), 3.0, dtype=dtype, device="cuda")
    status = u.status_word()
    rows = torch.tensor([9, 10, 2 ** 30, 0, -2 ** 31], dtype=torch.int32, device="cuda")
    u.ut_qk_norm_rope_fwd(q, k, rope, rows=rows, k_out=cache[:10], status=status)
    with pytest.raises(u.UtError, match="invalid argument"):
        u.check_status(status)
    want = u.ut_qk_norm_rope_fwd(q, k, rope)[1]
    assert torch.equal(cache[9], want[0]) and torch.equal(cache[0], want[3])
    assert bool((cache[1:9] == 3).all()) and bool((cache[10:] == 3).all())


@BOTH
def test_in_place(u, dtype):
    q, k, v, wq, wk, dqo, dko = inputs(200, 6, 3, 128, dtype, seed=7)
    rope, _ = rope_of(u, "canvas", 128)
    how = dict(wq=wq, wk=wk)
    want = u.ut_qk_norm_rope_fwd(q, k, rope, v=v, **how)
    grads = u.ut_qk_norm_rope_bwd(q, k, rope, dqo, dko, **how)
    g2 = u.ut_qk_norm_rope_bwd(q, k, rope, dqo, dko, dq=dqo, dk=dko, **how)
    assert g2[0] is dqo and all(torch.equal(a, b) for a, b in zip(grads, g2))
    got = u.ut_qk_norm_rope_fwd(q, k, rope, v=v, q_out=q, k_out=k, v_out=v, **how)
    assert got[0] is q and all(torch.equal(a, b) for a, b in zip(want, got))


@BOTH
def test_strided_outputs_leave_the_rest(u, dtype):
    q, k, v, wq, wk, dqo, dko = inputs(50, 4, 2, 64, dtype, seed=8)
    rope, _ = rope_of(u, "line", 64)
    e = 16 // torch.empty(0, dtype=dtype).element_size()
    buf = torch.full((52, 8 * 64 + 2 * e), 7.0, dtype=dtype, device="cuda")
    body = buf[1:-1, e:-e].unflatten(1, (8, 64))
    out = u.ut_qk_norm_rope_fwd(q, k, rope, v=v, wq=wq, wk=wk, q_out=body[:, :4], k_out=body[:, 4:6], v_out=body[:, 6:])
    want = u.ut_qk_norm_rope_fwd(q.contiguous(), k.contiguous(), rope, v=v.contiguous(), wq=wq, wk=wk)
    assert all(torch.equal(a, b) for a, b in zip(out, want))
    grads = u.ut_qk_norm_rope_bwd(q, k, rope, dqo, dko, wq=wq, wk=wk, dq=body[:, :4], dk=body[:, 4:6])
    assert all(torch.equal(a, b) for a, b in zip(grads, u.ut_qk_norm_rope_bwd(q, k, rope, dqo, dko, wq=wq, wk=wk)))
    frame = buf.clone()
    frame[1:-1, e:-e] = 7.0
    assert torch.equal(frame, torch.full_like(buf, 7.0))


@BOTH
def test_no_rows(u, dtype):
    q, k, v, wq, wk, dqo, dko = inputs(0, 4, 2, 64, dtype)
    rope, _ = rope_of(u, "line", 64)
    out = u.ut_qk_norm_rope_fwd(q, k, rope, v=v, wq=wq, wk=wk)
    assert [t.shape[0] for t in out] == [0, 0, 0]
    dq, dk, dwq, dwk = u.ut_qk_norm_rope_bwd(q, k, rope, dqo, dko, wq=wq, wk=wk)
    assert dq.shape == q.shape and not dwq.any() and not dwk.any()


@BOTH
def test_same_bits_on_every_run_stream_and_graph(u, dtype):
    x = inputs(900, 6, 2, 128, dtype, seed=9)
    q, k, v, wq, wk, dqo, dko = x
    rope, _ = rope_of(u, "canvas", 128)

    def both():
        return (*u.ut_qk_norm_rope_fwd(q, k, rope, v=v, wq=wq, wk=wk),
                *u.ut_qk_norm_rope_bwd(q, k, rope, dqo, dko, wq=wq, wk=wk))

    first = both()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = both()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        captured = both()
    for _ in range(2):
        g.replay()
    torch.cuda.synchronize()
    for other in (again, captured):
        assert all(torch.equal(a, b) for a, b in zip(first, other))


def test_gradient_matches_differences(u):
    x = inputs(40, 4, 2, 64, torch.float32, seed=10)
    q, k, v, wq, wk, dqo, dko = x
    rope, args = rope_of(u, "line", 64)
    grads = u.ut_qk_norm_rope_bwd(q, k, rope, dqo, dko, wq=wq, wk=wk, eps=EPS)
    ang = o.angles(range(40), *args)
    g = np.random.Generator(np.random.PCG64(2))
    for a, w, dy, dx, dw in ((q, wq, dqo, grads[0], grads[2]), (k, wk, dko, grads[1], grads[3])):
        a, w, dy = to_np(a), to_np(w), to_np(dy)
        f = lambda s, t: (o.qk_norm_rope(s, t, EPS, ang)[0] * dy).sum()  # noqa: E731
        for got, d, at in ((dx, g.standard_normal(a.shape), 0), (dw, g.standard_normal(w.shape), 1)):
            h = 1e-5
            want = (f(a + h * d, w) - f(a - h * d, w) if at == 0 else f(a, w + h * d) - f(a, w - h * d)) / (2 * h)
            terms = np.abs(to_np(got) * d).sum()
            assert abs((to_np(got) * d).sum() - want) <= 2.0 ** -15 * terms + 1e-6


def test_as_the_rotated_gather(u):
    """Heads of norm one: the rotation is that of ut_fg_gather_rope (bf16, each result rounded once)."""
    x = torch.randn(100, 4, 128, generator=torch.Generator().manual_seed(11)).cuda()
    x = (x / x.square().mean(-1, keepdim=True).sqrt()).bfloat16()
    idx = torch.arange(100, dtype=torch.int32, device="cuda")
    rope = u.rope_config(6, (16, 56, 56), 10000.0, 9)
    want = u.ut_fg_gather_rope(idx, 100, [x], rope)[0].float()
    got = u.ut_qk_norm_rope_fwd(x, x, rope, pos=idx)[0].float()
    # the norm of a rounded head is one to 2^-8, and both results are rounded
    pair = (x.float()[..., 0::2].abs() + x.float()[..., 1::2].abs()).repeat_interleave(2, -1)
    assert bool(((got - want).abs() <= 2.0 ** -8 * (want.abs() * 2 + pair * 1.01)).all())

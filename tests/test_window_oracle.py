"""The float64 definitions of the windowed-attention operators against torch in float64, loops and differences."""
import numpy as np
import pytest
import torch

import oracle.window_oracle as o


def rng(seed):
    return np.random.Generator(np.random.PCG64(seed))


def prefix(lengths):
    return np.concatenate([[0], np.cumsum(lengths)])


@pytest.mark.parametrize("n_q,n_k,win", [(5, 5, (1, 0, 0)), (3, 9, (2, 1, 2)), (7, 4, (100, 0, 0)), (1, 6, (0, 0, 3)),
                                         (4, 0, (1, 1, 1)), (6, 6, (0, 9, 0))])
def test_seen_keys(n_q, n_k, win):
    left, right, sinks = win
    got = o.seen(n_q, n_k, *win)
    assert got.shape == (n_q, n_k)
    for i in range(n_q):
        p = n_k - n_q + i
        for j in range(n_k):
            behind, near, first = j > p + right, j >= p - left, j < sinks
            assert got[i, j] == (not behind and (near or first))


@pytest.mark.parametrize("heads,kv_heads,win", [(1, 1, (2, 0, 1)), (6, 2, (1, 2, 0)), (4, 1, (50, 50, 0))])
def test_attention_matches_torch(heads, kv_heads, win):
    g = rng(1)
    cu_q, cu_k, k_len = prefix([3, 0, 5]), prefix([6, 2, 7]), [4, 1, 7]
    q, dout = g.standard_normal((8, heads, 64)), g.standard_normal((8, heads, 64))
    k, v = g.standard_normal((15, kv_heads, 64)), g.standard_normal((15, kv_heads, 64))
    mask = np.ones(15, np.uint8)
    mask[[1, 12]] = 0
    tq, tk, tv = (torch.tensor(x, requires_grad=True) for x in (q, k, v))
    outs = []
    for s in range(3):
        n, m = cu_q[s + 1] - cu_q[s], k_len[s]
        keys = slice(cu_k[s], cu_k[s] + m)
        on = torch.tensor([[j <= m - n + i + win[1] and (j >= m - n + i - win[0] or j < win[2]) and mask[cu_k[s] + j] != 0
                            for j in range(m)] for i in range(n)]).reshape(n, m)
        assert bool(on.any(1).all())
        a = [tq[cu_q[s]:cu_q[s + 1]]] + [t[keys].repeat_interleave(heads // kv_heads, 1) for t in (tk, tv)]
        outs.append(torch.nn.functional.scaled_dot_product_attention(
            *(t.transpose(0, 1) for t in a), attn_mask=on).transpose(0, 1))
    want = torch.cat(outs)
    got, lse, _ = o.window_fwd(q, k, v, cu_q, cu_k, win, k_len, mask)
    assert np.abs(got - want.detach().numpy()).max() < 1e-12 and np.isfinite(lse).all()
    grads = torch.autograd.grad(want, (tq, tk, tv), torch.tensor(dout))
    r = o.window_bwd(q, k, v, dout, cu_q, cu_k, win, k_len, mask)
    for name, t in zip(("dq", "dk", "dv"), grads):
        assert np.abs(r[name] - t.numpy()).max() < 1e-12, name
    for name in ("dk", "dv"):
        assert not r[name][mask == 0].any() and not r[name][4:6].any() and not r[name][7:8].any()


def test_rows_without_keys():
    g = rng(2)
    q, k = g.standard_normal((4, 2, 64)), g.standard_normal((2, 2, 64))
    got, lse, _ = o.window_fwd(q, k, k, prefix([4]), prefix([2]), (5, 0, 1))
    assert not got[:2].any() and np.all(np.isneginf(lse[:, :2])) and np.isfinite(lse[:, 2:]).all()
    r = o.window_bwd(q, k, k, q, prefix([4]), prefix([2]), (5, 0, 1))
    assert not r["dq"][:2].any() and all(np.isfinite(x).all() for x in r.values())


def test_attention_gradient_matches_differences():
    g = rng(3)
    cu, win, h = prefix([7, 4]), (2, 1, 1), 1e-5
    x = [g.standard_normal(s) for s in ((11, 4, 64), (11, 2, 64), (11, 2, 64))]
    dout = g.standard_normal((11, 4, 64))
    r = o.window_bwd(*x, dout, cu, cu, win)
    for i, name in enumerate(("dq", "dk", "dv")):
        d = g.standard_normal(x[i].shape)
        up, down = ([y + t * h * d if j == i else y for j, y in enumerate(x)] for t in (1, -1))
        want = ((o.window_fwd(*up, cu, cu, win)[0] - o.window_fwd(*down, cu, cu, win)[0]) * dout).sum() / (2 * h)
        assert abs((r[name] * d).sum() - want) < 1e-7 * max(1, abs(want)), name


def test_norm_matches_a_loop():
    g = rng(4)
    x, w, pos = g.standard_normal((3, 2, 64)), g.standard_normal(64), [3, 700, -5]
    axes, side, prefix_ = (8, 28, 28), 5, 12
    ang = o.angles(pos, side, axes, 10000.0, prefix_)
    got, _ = o.qk_norm_rope(x, w, 1e-6, ang)
    for n in range(3):
        t = max(0, pos[n] - prefix_)
        where = (t // 25, t % 25 // 5, t % 5)
        for h in range(2):
            y = x[n, h] / np.sqrt(np.mean(x[n, h] ** 2) + 1e-6) * w
            e = 0
            for a in range(3):
                for j in range(axes[a] // 2):
                    z = complex(y[2 * e], y[2 * e + 1]) * np.exp(1j * where[a] * 10000.0 ** (-2 * j / axes[a]))
                    assert abs(complex(got[n, h, 2 * e], got[n, h, 2 * e + 1]) - z) < 1e-12
                    e += 1


def test_norm_gradient_matches_differences():
    g = rng(5)
    x, w, dy = g.standard_normal((4, 3, 64)), g.standard_normal(64), g.standard_normal((4, 3, 64))
    ang = o.angles([0, 9, 77, 1234], 1, (64, 0, 0), 10000.0, 0)
    dx, dw, dx_abs, dw_abs = o.qk_norm_rope_bwd(x, w, 1e-6, ang, dy)
    h = 1e-6
    f = lambda a, b: (o.qk_norm_rope(a, b, 1e-6, ang)[0] * dy).sum()  # noqa: E731
    d, e = g.standard_normal(x.shape), g.standard_normal(64)
    assert abs((dx * d).sum() - (f(x + h * d, w) - f(x - h * d, w)) / (2 * h)) < 1e-6
    assert abs((dw * e).sum() - (f(x, w + h * e) - f(x, w - h * e)) / (2 * h)) < 1e-6
    assert np.all(np.abs(dx) <= dx_abs + 1e-12) and np.all(np.abs(dw) <= dw_abs + 1e-12)

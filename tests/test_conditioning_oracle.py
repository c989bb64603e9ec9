"""The float64 definitions of the conditioning operators against torch in float64 and against central differences."""
import numpy as np
import pytest
import torch

import oracle.conditioning_oracle as o


def rng(seed):
    return np.random.Generator(np.random.PCG64(seed))


@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (6, 2)])
def test_cross_attention_matches_torch(heads, kv_heads):
    g = rng(1)
    cu_q, cu_k = o.prefix([3, 0, 5]), o.prefix([4, 2, 7])
    q, dout = g.standard_normal((8, heads, 64)), g.standard_normal((8, heads, 64))
    k, v = g.standard_normal((13, kv_heads, 64)), g.standard_normal((13, kv_heads, 64))
    mask = np.ones(13, np.uint8)
    mask[[1, 8, 12]] = 0
    tq, tk, tv = (torch.tensor(x, requires_grad=True) for x in (q, k, v))
    outs = []
    for s in range(3):
        keys = [j for j in range(cu_k[s], cu_k[s + 1]) if mask[j]]
        a = [tq[cu_q[s]:cu_q[s + 1]]] + [t[keys].repeat_interleave(heads // kv_heads, 1) for t in (tk, tv)]
        outs.append(torch.nn.functional.scaled_dot_product_attention(*(t.transpose(0, 1) for t in a)).transpose(0, 1))
    want = torch.cat(outs)
    got, lse, _ = o.xattn_fwd(q, k, v, cu_q, cu_k, mask)
    assert np.abs(got - want.detach().numpy()).max() < 1e-12
    grads = torch.autograd.grad(want, (tq, tk, tv), torch.tensor(dout))
    r = o.xattn_bwd(q, k, v, dout, cu_q, cu_k, mask)
    for name, t in zip(("dq", "dk", "dv"), grads):
        assert np.abs(r[name] - t.numpy()).max() < 1e-12, name
    assert not r["dk"][mask == 0].any() and not r["dv"][mask == 0].any()


def test_cross_attention_rows_without_keys():
    g = rng(2)
    q, k, v = g.standard_normal((4, 2, 64)), g.standard_normal((3, 2, 64)), g.standard_normal((3, 2, 64))
    got, lse, _ = o.xattn_fwd(q, k, v, o.prefix([2, 2]), o.prefix([0, 3]), np.zeros(3, np.uint8))
    assert not got.any() and np.all(np.isneginf(lse))
    one, lse1, _ = o.xattn_fwd(q, k[:1], v[:1], o.prefix([4]), o.prefix([1]))
    assert np.allclose(one, v[0]) and np.allclose(lse1, 64 ** -0.5 * np.einsum("nhd,hd->hn", q, k[0]))


def test_cross_attention_gradient_matches_differences():
    g = rng(3)
    cu_q, cu_k = o.prefix([3, 2]), o.prefix([4, 5])
    x = [g.standard_normal(s) for s in ((5, 4, 64), (9, 2, 64), (9, 2, 64))]
    dout = g.standard_normal((5, 4, 64))
    r = o.xattn_bwd(*x, dout, cu_q, cu_k)
    h = 1e-5
    for i, name in enumerate(("dq", "dk", "dv")):
        d = g.standard_normal(x[i].shape)
        up, down = ([y + t * h * d if j == i else y for j, y in enumerate(x)] for t in (1, -1))
        want = ((o.xattn_fwd(*up, cu_q, cu_k)[0] - o.xattn_fwd(*down, cu_q, cu_k)[0]) * dout).sum() / (2 * h)
        assert abs((r[name] * d).sum() - want) < 1e-7 * max(1, abs(want)), name


@pytest.mark.parametrize("act", [0, 1])
@pytest.mark.parametrize("channels,groups", [(12, 4), (8, 8), (6, 1)])
def test_group_norm_matches_torch_and_differences(act, channels, groups):
    g = rng(4)
    cu = o.prefix([5, 0, 1, 7])
    x, dy = g.standard_normal((13, channels)) + 3, g.standard_normal((13, channels))
    gamma, beta = g.standard_normal(channels), g.standard_normal(channels)
    tx, tg, tb = (torch.tensor(t, requires_grad=True) for t in (x, gamma, beta))
    outs = []
    for s in range(4):
        if cu[s] == cu[s + 1]:
            continue
        t = tx[cu[s]:cu[s + 1]].t()[None]
        if channels // groups * t.shape[2] == 1:  # a single value: torch refuses it, and the value itself is beta
            outs.append((tx[cu[s]:cu[s + 1]] * 0 + tb + 0 * tg))
        else:
            outs.append(torch.nn.functional.group_norm(t, groups, tg, tb, 1e-5)[0].t())
    u = torch.cat(outs)
    want = torch.nn.functional.silu(u) if act else u
    y, mean, rstd = o.group_norm_fwd(x, gamma, beta, groups, 1e-5, act, cu)
    assert np.abs(y - want.detach().numpy()).max() < 1e-11
    assert np.allclose(rstd[1], 1e5 ** 0.5) and not mean[1].any()
    r = o.group_norm_bwd(x, dy, gamma, beta, groups, 1e-5, act, cu)
    for name, t in zip(("dx", "dgamma", "dbeta"), torch.autograd.grad(want, (tx, tg, tb), torch.tensor(dy))):
        assert np.abs(r[name] - t.numpy()).max() < 1e-9, name
    h, d = 1e-6, g.standard_normal(x.shape)
    f = [o.group_norm_fwd(x + t * h * d, gamma, beta, groups, 1e-5, act, cu)[0] for t in (1, -1)]
    want = ((f[0] - f[1]) * dy).sum() / (2 * h)
    assert abs((r["dx"] * d).sum() - want) < 1e-6 * max(1, abs(want))

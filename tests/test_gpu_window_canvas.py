"""The windowed block on a canvas: the tokens that a compaction retains, rotated by their canvas positions, against the
float64 definitions, and the same tokens through a cache.

Tolerances: those of the windowed block's tests (fp32: 2^-9 of a tensor's largest magnitude; bf16: a relative root mean
square of 2e-2), for the same stages."""
import numpy as np
import pytest
import torch

import oracle.window_oracle as o
from gpu_util import need_gpu, to_np
from test_gpu_window_block import BOTH, near

pytestmark = pytest.mark.gpu
H, HK, D, C, EPS = 4, 2, 64, 96, 1e-6
SIDE, IMAGES, TEXT, AXES = 8, 3, 20, (8, 28, 28)


@pytest.fixture(scope="module")
def u():
    need_gpu()
    from paper_2609_23169_gb300 import ultratex
    return ultratex


def retained(u, dtype):
    """(x [n, C], positions [n], weights, dy [n, C]) of a canvas whose background tokens are dropped."""
    from paper_2609_23169_gb300.window import WindowWeights
    g = torch.Generator().manual_seed(90)

    def normal(*shape, scale=1.0):
        return (torch.randn(*shape, generator=g) * scale).to(dtype).cuda()

    w = WindowWeights(normal((H + 2 * HK) * D, C, scale=C ** -0.5), (1 + 0.2 * torch.randn(D, generator=g)).cuda(),
                      (1 + 0.2 * torch.randn(D, generator=g)).cuda(), normal(C, H * D, scale=(H * D) ** -0.5))
    t = TEXT + IMAGES * SIDE * SIDE
    mask = (torch.rand(t, generator=g) < 0.6).to(torch.uint8)
    mask[:TEXT] = 1
    idx, n, (x,) = u.ut_fg_compact(mask.cuda(), [normal(t, C)])
    n = int(n.item())
    return x[:n], idx[:n], w, normal(n, C)


def stages(x, w, idx, win):
    n = x.shape[0]
    x, wqkv, nq, nk, wo = (to_np(t).astype(np.float64) for t in (x, w.wqkv, w.norm_q, w.norm_k, w.wo))
    qkv = (x @ wqkv.T).reshape(n, H + 2 * HK, D)
    q, k, v = qkv[:, :H], qkv[:, H:H + HK], qkv[:, H + HK:]
    ang = o.angles(idx.tolist(), SIDE, AXES, 10000.0, TEXT)
    qn, kn = o.qk_norm_rope(q, nq, EPS, ang)[0], o.qk_norm_rope(k, nk, EPS, ang)[0]
    att = o.window_fwd(qn, kn, v, [0, n], [0, n], win)[0]
    return x, wqkv, nq, nk, wo, q, k, v, ang, qn, kn, att, x + att.reshape(n, -1) @ wo.T


@BOTH
@pytest.mark.parametrize("win", [(30, 30, TEXT), (15, 0, 4)])
def test_training_step(u, win, dtype):
    from paper_2609_23169_gb300.window import WindowBlock
    x, idx, w, dy = retained(u, dtype)
    n = x.shape[0]
    block = WindowBlock(H, HK, D, u.rope_config(SIDE, AXES, 10000.0, TEXT), *win, eps=EPS)
    status = u.status_word()
    y = block.forward(x, w, pos=idx, status=status)
    dx, dw = block.backward(dy)
    u.check_status(status)
    hx, wqkv, nq, nk, wo, q, k, v, ang, qn, kn, att, want = stages(x, w, idx, win)
    hdy = to_np(dy).astype(np.float64)
    r = o.window_bwd(qn, kn, v, (hdy @ wo).reshape(n, H, D), [0, n], [0, n], win)
    dq, dnq = o.qk_norm_rope_bwd(q, nq, EPS, ang, r["dq"])[:2]
    dk, dnk = o.qk_norm_rope_bwd(k, nk, EPS, ang, r["dk"])[:2]
    dqkv = np.concatenate([dq, dk, r["dv"]], axis=1).reshape(n, -1)
    refs = (want, hdy + dqkv @ wqkv, dqkv.T @ hx, dnq, dnk, hdy.T @ att.reshape(n, -1))
    for got, ref, what in zip((y, dx, dw.wqkv, dw.norm_q, dw.norm_k, dw.wo), refs, ("y", "dx", "wqkv", "nq", "nk", "wo")):
        near(got, torch.tensor(ref), dtype, what)


@BOTH
def test_through_a_cache(u, dtype):
    from paper_2609_23169_gb300.window import WindowBlock, WindowCache
    x, idx, w, _ = retained(u, dtype)
    n, win = x.shape[0], (15, 0, 4)
    block = WindowBlock(H, HK, D, u.rope_config(SIDE, AXES, 10000.0, TEXT), *win, eps=EPS)
    cache = WindowCache(1, n, HK, D, dtype)
    got, at = [], 0
    for c in (TEXT + 3, 1, 1, n - TEXT - 5):
        cu = torch.tensor([0, c], dtype=torch.int32, device="cuda")
        got.append(block.extend(x[at:at + c], w, cache, cu, pos=idx[at:at + c]))
        at += c
    u.check_status(cache.status)
    assert at == n
    near(torch.cat(got), torch.tensor(stages(x, w, idx, win)[-1]), dtype, "y")

"""The windowed block (projection, norms with rotation, windowed attention, projection) against float64: training over
packed segments, and the same tokens fed through caches.

Tolerances, derived before the first run.  fp32: each of the four stages carries at most 2^-16 of its terms' magnitudes
(the operators' own bound); the terms of a projection of up to 384 values exceed its result by up to about 20, so
results are within 4 x 20 x 2^-16 < 2^-9 of the largest magnitude of their tensor.  bf16: every stage rounds its result
once (2^-9 relative, root mean square), a gradient passes through eight of them: within the relative root mean square
that the bf16 attention outputs have, 2e-2."""
import numpy as np
import pytest
import torch

from gpu_util import BF16_REL_RMS, err_stats, need_gpu, to_np

pytestmark = pytest.mark.gpu

H, HK, D, C = 4, 2, 64, 96
LENGTHS, WIN = [70, 0, 33, 150], (40, 0, 5)
EPS = 1e-6
BOTH = pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])


@pytest.fixture(scope="module")
def u():
    need_gpu()
    from paper_2609_23169_gb300 import ultratex
    return ultratex


def inputs(dtype):
    from paper_2609_23169_gb300.window import WindowWeights
    g = torch.Generator().manual_seed(5)

    def normal(*shape, scale=1.0):
        return (torch.randn(*shape, generator=g) * scale).to(dtype).cuda()

    w = WindowWeights(normal((H + 2 * HK) * D, C, scale=C ** -0.5), (1 + 0.2 * torch.randn(D, generator=g)).cuda(),
                      (1 + 0.2 * torch.randn(D, generator=g)).cuda(), normal(C, H * D, scale=(H * D) ** -0.5))
    n = sum(LENGTHS)
    pos = torch.cat([torch.arange(x) for x in LENGTHS]).int()
    cu = torch.tensor(np.concatenate([[0], np.cumsum(LENGTHS)]), dtype=torch.int32)
    return normal(n, C), w, pos.cuda(), cu.cuda(), normal(n, C)


def plain(x, w, pos, cu, dy, mask=None):
    """The block in float64 torch, its gradients by automatic differentiation."""
    x, dy = x.double().cpu().requires_grad_(), dy.double().cpu()
    p = [t.double().cpu().requires_grad_() for t in (w.wqkv, w.norm_q, w.norm_k, w.wo)]
    n = x.shape[0]
    qkv = (x @ p[0].t()).view(n, H + 2 * HK, D)
    ang = pos.double().cpu()[:, None] * 10000.0 ** (-2.0 * torch.arange(D // 2).double() / D)
    turn = torch.polar(torch.ones_like(ang), ang)[:, None]

    def norm(t, wt):
        t = t * torch.rsqrt(t.square().mean(-1, keepdim=True) + EPS) * wt
        return torch.view_as_real(torch.view_as_complex(t.reshape(n, -1, D // 2, 2)) * turn).reshape(n, -1, D)

    q, k, v = norm(qkv[:, :H], p[1]), norm(qkv[:, H:H + HK], p[2]), qkv[:, H + HK:]
    o, at = [], cu.cpu().tolist()
    for a, b in zip(at, at[1:]):
        i, j = torch.arange(b - a)[:, None], torch.arange(b - a)[None]
        on = (j <= i + WIN[1]) & ((j >= i - WIN[0]) | (j < WIN[2]))
        if mask is not None:
            on = on & mask.cpu()[a:b].bool()
        for h in range(H):
            s = (q[a:b, h] @ k[a:b, h // (H // HK)].t() / D ** 0.5).masked_fill(~on, -torch.inf)
            pr = torch.where(on.any(1, keepdim=True), torch.softmax(torch.where(on.any(1, keepdim=True), s, 0.0), 1), 0.0)
            o.append((a, b, h, pr @ v[a:b, h // (H // HK)]))
    att = torch.zeros(n, H, D, dtype=torch.float64)
    for a, b, h, t in o:
        att = att.index_put((torch.arange(a, b), torch.tensor(h)), t)
    y = x + att.flatten(1) @ p[3].t()
    return [y.detach()] + list(torch.autograd.grad(y, [x] + p, dy))


def near(got, ref, dtype, what):
    s = err_stats(to_np(got), to_np(ref))
    if dtype == torch.float32:
        assert s["max_abs"] <= 2.0 ** -9 * float(ref.abs().max()), (what, s)
    else:
        assert s["rel_rms"] <= BF16_REL_RMS, (what, s)


@BOTH
@pytest.mark.parametrize("masked", [False, True])
def test_training_step(u, masked, dtype):
    from paper_2609_23169_gb300.window import WindowBlock
    x, w, pos, cu, dy = inputs(dtype)
    mask = None
    if masked:
        mask = (torch.rand(x.shape[0], generator=torch.Generator().manual_seed(6)) < 0.8).to(torch.uint8).cuda()
    block = WindowBlock(H, HK, D, u.rope_config(1, (D, 0, 0)), *WIN, eps=EPS)
    status = u.status_word()
    y = block.forward(x, w, pos=pos, cu=cu, key_mask=mask, status=status)
    dx, dw = block.backward(dy)
    u.check_status(status)
    want = plain(x, w, pos, cu, dy, mask)
    for got, ref, what in zip((y, dx, dw.wqkv, dw.norm_q, dw.norm_k, dw.wo), want, ("y", "dx", "wqkv", "nq", "nk", "wo")):
        near(got, ref, dtype, what)


@BOTH
def test_caches_give_what_training_gives(u, dtype):
    """Prompts of each segment, then single tokens, one segment pausing in between: the outputs of the whole sequence."""
    from paper_2609_23169_gb300.window import WindowBlock, WindowCache
    x, w, pos, cu, _ = inputs(dtype)
    block = WindowBlock(H, HK, D, u.rope_config(1, (D, 0, 0)), *WIN, eps=EPS)
    cache = WindowCache(len(LENGTHS), 160, HK, D, dtype)
    want = plain(x, w, pos, cu, x)[0]
    status = u.status_word()
    done, got = [0] * len(LENGTHS), torch.empty_like(x)
    at = cu.tolist()
    for chunk in ([60, 0, 1, 1], [1, 0, 1, 130], [1, 0, 0, 1], [1, 0, 1, 1], [7, 0, 30, 17]):
        take = [torch.arange(at[s] + done[s], at[s] + done[s] + c) for s, c in enumerate(chunk)]
        rows = torch.cat(take).cuda()
        cu_q = torch.tensor(np.concatenate([[0], np.cumsum(chunk)]), dtype=torch.int32, device="cuda")
        got[rows] = block.extend(x[rows], w, cache, cu_q, status=status)
        done = [a + b for a, b in zip(done, chunk)]
    u.check_status(status)
    assert done == LENGTHS and cache.length.tolist() == LENGTHS
    near(got, want, dtype, "y")


def test_single_tokens_in_a_graph(u):
    """A captured step, replayed: each replay appends a token to every cache."""
    from paper_2609_23169_gb300.window import WindowBlock, WindowCache
    x, w, pos, cu, _ = inputs(torch.bfloat16)
    block = WindowBlock(H, HK, D, u.rope_config(1, (D, 0, 0)), *WIN, eps=EPS)
    eager, graphed = (WindowCache(3, 64, HK, D) for _ in range(2))
    cu_q = torch.arange(4, dtype=torch.int32, device="cuda")
    step = torch.empty(3, C, dtype=torch.bfloat16, device="cuda")
    step.copy_(x[:3])
    block.extend(step, w, graphed, cu_q)  # warm-up
    graphed.length.zero_()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = block.extend(step, w, graphed, cu_q)
    graphed.length.zero_()
    for i in range(50):
        step.copy_(x[3 * i:3 * i + 3])
        g.replay()
        want = block.extend(step, w, eager, cu_q)
        assert torch.equal(out, want), i
    assert torch.equal(eager.k, graphed.k) and graphed.length.tolist() == [50] * 3


def test_a_full_cache_is_reported(u):
    from paper_2609_23169_gb300.window import WindowBlock, WindowCache
    x, w, _, _, _ = inputs(torch.bfloat16)
    block = WindowBlock(H, HK, D, u.rope_config(1, (D, 0, 0)), *WIN, eps=EPS)
    cache = WindowCache(2, 4, HK, D)
    cu_q = torch.tensor([0, 3, 8], dtype=torch.int32, device="cuda")
    status = u.status_word()
    block.extend(x[:8], w, cache, cu_q, status=status)
    with pytest.raises(u.UtError, match="invalid argument"):
        u.check_status(status)

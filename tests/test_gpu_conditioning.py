"""The conditioning block over retained tokens (group norm + SiLU, projections, cross attention) against float64, and
the bounded waits of its kernels.

Tolerances, derived before the first run.  fp32: each of the five stages carries at most 2^-17 of its terms'
magnitudes (the operators' own bound); the terms of a projection of up to 200 values exceed its result by up to about
16, so results are within 5 x 16 x 2^-17 < 2^-10 of the largest magnitude of their tensor.  bf16: every stage rounds
its result once (2^-9 relative, root mean square), the gradients pass through eight of them: within the relative root
mean square that the bf16 attention outputs have, 2e-2."""
import numpy as np
import pytest
import torch

from gpu_util import BF16_REL_RMS, err_stats, need_gpu, to_np

pytestmark = pytest.mark.gpu

IMAGES, TOKENS, H, HK, D, GROUPS, C, E = 4, 60, 4, 2, 64, 8, 96, 40
PROMPTS = [9, 0, 130, 21]


@pytest.fixture(scope="module")
def u():
    need_gpu()
    from paper_2609_23169_gb300 import ultratex
    return ultratex


def inputs(dtype):
    g = torch.Generator().manual_seed(5)

    def normal(*shape, scale=1.0):
        return (torch.randn(*shape, generator=g) * scale).to(dtype).cuda()

    mask = (torch.rand(IMAGES * TOKENS, generator=g) < 0.6).to(torch.uint8)
    mask[2 * TOKENS:3 * TOKENS - 1] = 0  # an image with one token at most
    mask[3 * TOKENS - 1] = 1
    M = sum(PROMPTS)
    key_mask = (torch.rand(M, generator=g) < 0.8).to(torch.uint8)
    cu = torch.tensor(np.concatenate([[0], np.cumsum(PROMPTS)]), dtype=torch.int32)
    from paper_2609_23169_gb300.conditioning import BlockWeights
    w = BlockWeights((1 + 0.2 * torch.randn(C, generator=g)).cuda(), (0.2 * torch.randn(C, generator=g)).cuda(),
                     normal(H * D, C, scale=C ** -0.5), normal(2 * HK * D, E, scale=E ** -0.5),
                     normal(C, H * D, scale=(H * D) ** -0.5))
    return mask.cuda(), normal(IMAGES * TOKENS, C), normal(M, E), cu.cuda(), key_mask.cuda(), w, \
        normal(IMAGES * TOKENS, C)


def plain(mask, x, states, cu, key_mask, w, dy):
    """The block in float64 torch, its gradients by automatic differentiation."""
    x, states, dy = (t.double().cpu() for t in (x, states, dy))
    p = [t.double().cpu().requires_grad_() for t in (w.gamma, w.beta, w.wq, w.wkv, w.wo)]
    gamma, beta, wq, wkv, wo = p
    x.requires_grad_()
    states.requires_grad_()
    keep, cu, mask = key_mask.cpu().bool(), cu.cpu().tolist(), mask.cpu().bool()
    y = x.clone()
    kv = (states @ wkv.t()).view(-1, 2, HK, D)
    for i in range(IMAGES):
        rows = torch.arange(i * TOKENS, (i + 1) * TOKENS)[mask[i * TOKENS:(i + 1) * TOKENS]]
        xr = x[rows]
        z = xr.view(-1, GROUPS, C // GROUPS)
        z = (z - z.mean((0, 2), keepdim=True)) / torch.sqrt(z.var((0, 2), unbiased=False, keepdim=True) + 1e-5)
        h = torch.nn.functional.silu(z.reshape(-1, C) * gamma + beta)
        keys = torch.arange(cu[i], cu[i + 1])[keep[cu[i]:cu[i + 1]]]
        if keys.numel():
            q = (h @ wq.t()).view(-1, H, D)
            k, v = (kv[keys, j].repeat_interleave(H // HK, 1) for j in (0, 1))
            o = torch.einsum("hij,jhd->ihd", torch.einsum("ihd,jhd->hij", q * D ** -0.5, k).softmax(-1), v)
            xr = xr + o.reshape(-1, H * D) @ wo.t()
        y = y.index_put((rows,), xr)
    y.backward(dy)
    return [t.detach().numpy() for t in (y, x.grad, states.grad, *(t.grad for t in p))]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_block_matches_float64(u, dtype):
    from paper_2609_23169_gb300.conditioning import ConditioningBlock
    mask, x, states, cu, key_mask, w, dy = inputs(dtype)
    block = ConditioningBlock(IMAGES, TOKENS, H, HK, D, GROUPS)
    status = u.status_word()
    y = block.forward(mask, x, states, cu, w, key_mask, status)
    dx, dstates, g = block.backward(dy, status)
    torch.cuda.synchronize()
    u.check_status(status)
    got = [y, dx, dstates, g.gamma, g.beta, g.wq, g.wkv, g.wo]
    ref = plain(mask, x, states, cu, key_mask, w, dy)
    for name, a, b in zip(("y", "dx", "dstates", "dgamma", "dbeta", "dwq", "dwkv", "dwo"), got, ref):
        s = err_stats(to_np(a), b)
        if dtype == torch.float32:
            assert s["max_abs"] <= 2.0 ** -10 * np.abs(b).max(), (name, s)
        else:
            assert s["rel_rms"] <= BF16_REL_RMS, (name, s)
    dropped = (mask == 0).cpu()
    assert torch.equal(y.cpu()[dropped], x.cpu()[dropped]) and torch.equal(dx.cpu()[dropped], dy.cpu()[dropped])


def test_image_prefix(u):
    from paper_2609_23169_gb300.conditioning import image_prefix
    idx = torch.tensor([0, 4, 10, 11, 12, 39], dtype=torch.int32, device="cuda")
    assert image_prefix(idx, 4, 10).tolist() == [0, 2, 5, 5, 6]
    assert image_prefix(idx[:0], 4, 10).tolist() == [0, 0, 0, 0, 0]


def test_expired_waits_report_timeout_and_context_survives(u, monkeypatch):
    """With the limit at 0 the waits run out: the kernels say so in the status word, end, and the next calls work.
    (The sizes are such that some warps wait for 100 us and more, or many times: the first try of a wait may itself take
    microseconds, so that a short one is met within it.)"""
    g = torch.Generator().manual_seed(6)
    q, do = (torch.randn(20480, 4, 128, generator=g).bfloat16().cuda() for _ in range(2))
    k, v = (torch.randn(16384, 2, 128, generator=g).bfloat16().cuda() for _ in range(2))
    x, dy = (torch.randn(400000, 320, generator=g).bfloat16().cuda() for _ in range(2))
    want = u.ut_xattn_fwd(q, k, v)
    want_g = u.ut_xattn_bwd(q, k, v, *want, do)
    want_n = u.ut_group_norm_fwd(x, None, None, 32)
    want_ng = u.ut_group_norm_bwd(x, dy, None, None, want_n[1], want_n[2], 32)
    calls = (lambda s: u.ut_xattn_fwd(q, k, v, status=s), lambda s: u.ut_xattn_bwd(q, k, v, *want, do, status=s),
             lambda s: u.ut_group_norm_fwd(x, None, None, 32, status=s),
             lambda s: u.ut_group_norm_bwd(x, dy, None, None, want_n[1], want_n[2], 32, status=s))
    monkeypatch.setenv("UT_WAIT_TIMEOUT_NS", "0")
    for f in calls:
        status = u.status_word()
        f(status)
        torch.cuda.synchronize()
        assert int(status.item()) == u.UT_ERR_TIMEOUT
    monkeypatch.delenv("UT_WAIT_TIMEOUT_NS")
    for f, ref in zip(calls, (want, want_g, want_n, want_ng)):
        status = u.status_word()
        got = f(status)
        torch.cuda.synchronize()
        assert int(status.item()) == 0
        for a, b in zip(got, ref):
            assert torch.equal(a, b)

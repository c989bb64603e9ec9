"""Key masks of windowed attention at d = 128, where two warps share a row's softmax, and where the keys are split, so
that whole parts have no key left.

Tolerances: those of the windowed attention tests, whose comparison with the float64 oracle is used."""
import ctypes

import pytest
import torch

from gpu_util import need_gpu, to_np
from test_gpu_window_attn import BOTH, check, i32, inputs, prefix

pytestmark = pytest.mark.gpu
HEADS = pytest.mark.parametrize("heads,kv_heads", [(2, 2), (6, 2)])
LENGTHS = [300, 40, 329]


@pytest.fixture(scope="module")
def u():
    need_gpu()
    from paper_2609_23169_gb300 import ultratex
    return ultratex


def mask_of(kind, n):
    mask = (torch.rand(n, generator=torch.Generator().manual_seed(1)) < 0.5).to(torch.uint8)
    if kind == "none_left":
        mask[:] = 0
    elif kind == "first_blocks":
        mask[:260] = 0
    elif kind == "only_last":
        mask[:] = 0
        mask[[299, 339, 668]] = 7
    elif kind == "half_blocks":  # the keys of one of the two warps of each block of a segment's first keys
        mask[:] = 1
        mask[64:128] = mask[340:404] = 0
    elif kind == "sinks_masked":
        mask[:9] = mask[300:309] = mask[340:349] = 0
    elif kind == "words":  # single bits at the borders of 32
        mask[:] = 0
        mask[[31, 32, 63, 64, 95, 96, 127, 128, 340 + 31, 340 + 64, 340 + 127]] = 1
    return mask


@BOTH
@HEADS
@pytest.mark.parametrize("win", [(70, 0, 9), (10, 30, 0), (500, 500, 0)])
@pytest.mark.parametrize("kind", ["random", "none_left", "first_blocks", "only_last", "half_blocks", "sinks_masked", "words"])
def test_masks(u, kind, win, heads, kv_heads, dtype):
    n = sum(LENGTHS)
    check(u, inputs(n, n, heads, kv_heads, 128, dtype, seed=70), LENGTHS, LENGTHS, win, mask=mask_of(kind, n).cuda())


@BOTH
def test_masked_and_foreign_rows_may_hold_anything(u, dtype):
    lengths, win = [170, 140, 230], (60, 20, 5)
    n = sum(lengths)
    q, k, v, dout = inputs(n, n, 4, 2, 128, dtype, seed=71)
    mask = (torch.rand(n, generator=torch.Generator().manual_seed(2)) < 0.6).to(torch.uint8).cuda()
    mask[170:310] = 1
    cu = i32(prefix(lengths))
    how = dict(left=win[0], right=win[1], sinks=win[2], cu_q=cu, cu_k=cu, key_mask=mask)
    clean = u.ut_window_attn_fwd(q, k, v, **how)
    grads = u.ut_window_attn_bwd(q, k, v, *clean, dout, **how)
    k2, v2, q2, dout2 = k.clone(), v.clone(), q.clone(), dout.clone()
    k2[mask == 0], v2[mask == 0] = float("nan"), float("inf")
    mid = slice(170, 310)  # the second segment is spoilt
    k2[mid], v2[mid], q2[mid], dout2[mid] = float("nan"), float("-inf"), float("inf"), float("nan")
    spoilt = u.ut_window_attn_fwd(q2, k2, v2, **how)
    grads2 = u.ut_window_attn_bwd(q2, k2, v2, *spoilt, dout2, **how)
    rest = torch.ones(n, dtype=torch.bool)
    rest[mid] = False
    assert torch.equal(clean[0][rest], spoilt[0][rest]) and torch.equal(clean[1][:, rest], spoilt[1][:, rest])
    for a, b in zip(grads, grads2):
        assert torch.equal(a[rest], b[rest])
    for g in grads2[1:]:
        assert not to_np(g)[rest.numpy() & (to_np(mask) == 0)].any()


@BOTH
def test_strides_and_odd_masks(u, dtype):
    """Slices of one projection and a mask at an odd address."""
    lengths, win = [45, 200], (130, 9, 3)
    q, k, v, dout = inputs(245, 245, 6, 3, 128, dtype, seed=72, fused=True, pad=8)
    mask = torch.ones(246, dtype=torch.uint8, device="cuda")[1:]
    mask[10:20] = mask[60:190] = 0
    check(u, (q, k, v, dout), lengths, lengths, win, mask=mask)


@BOTH
@pytest.mark.parametrize("heads,kv_heads", [(6, 2), (4, 4)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [1, 3])
def test_split_keys(u, n, d, heads, kv_heads, dtype):
    """New tokens over caches whose keys are split over blocks: masks that leave parts of them without a key, some rows
    without any, and NaN in all masked rows."""
    caps, k_len = [4000, 4000, 4000], [3990, 4000, 2500]
    lq = [n, n, n]
    q, k, v, dout = inputs(3 * n, 12000, heads, kv_heads, d, dtype, seed=73)
    mask = torch.zeros(12000, dtype=torch.uint8)
    mask[:12000:3] = 1
    mask[600:2900] = 0          # whole parts of the first segment
    mask[4000:8000] = 0         # of the second nothing,
    mask[8000:10400] = 0        # of the third its last keys
    if n > 1:
        mask[4005] = 1          # or one key, which all its rows see
    k[mask == 0], v[mask == 0] = float("nan"), float("inf")
    clean = (q, torch.where((mask != 0).cuda()[:, None, None], k, 0), torch.where((mask != 0).cuda()[:, None, None], v, 0), dout)
    for win in ((3999, 0, 0), (3000, 0, 130), (200, 0, 40)):
        out, lse, grads = check(u, clean, lq, caps, win, k_len=k_len, mask=mask.cuda())
        how = dict(left=win[0], right=win[1], sinks=win[2], k_len=i32(k_len), cu_q=i32(prefix(lq)), cu_k=i32(prefix(caps)),
                   key_mask=mask.cuda())
        out2, lse2 = u.ut_window_attn_fwd(q, k, v, **how)
        assert torch.equal(out, out2) and torch.equal(lse, lse2)
        for a, b in zip(grads, u.ut_window_attn_bwd(q, k, v, out2, lse2, dout, **how)):
            assert torch.equal(a, b)
    shape = u._xattn_shape(q, k, v, i32(prefix(lq)), i32(prefix(caps)), None, None)
    need = u.lib().ut_window_attn_fwd_workspace_size(ctypes.byref(shape), ctypes.byref(u.Window(3999, 0, 0)))
    assert need > 0  # the widest of the windows is split


@BOTH
@pytest.mark.parametrize("d", [64, 128])
def test_all_of_a_split_cache_masked(u, d, dtype):
    q, k, v, dout = inputs(2, 6000, 4, 2, d, dtype, seed=74)
    check(u, (q, k, v, dout), [2], [6000], (5999, 0, 4), mask=torch.zeros(6000, dtype=torch.uint8).cuda())

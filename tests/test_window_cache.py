"""What a full ``WindowCache`` does: a segment without room for all of its new tokens takes none of them, says so, and
leaves the other segments and every later call right.  On the CPU with float64 stand-ins for the two operators, and with
the operators themselves.

Tolerances: calls are compared with the same tokens in caches that are large enough.  A projection of fewer rows may add
its products in another order.  float64: that order alone, below 2^-40 of values of order one.  bf16: such a difference
turns single roundings of 2^-9 (root mean square) in eight stages, within the relative root mean square that the bf16
attention outputs have, 2e-2."""
import numpy as np
import pytest
import torch

import oracle.window_oracle as o
from gpu_util import BF16_REL_RMS, err_stats, to_np
from paper_2609_23169_gb300 import ultratex as u
from paper_2609_23169_gb300.window import WindowBlock, WindowCache, WindowWeights

H, HK, D, C = 4, 2, 64, 96
BOTH = pytest.mark.parametrize("device", ["cpu", pytest.param("cuda", marks=pytest.mark.gpu)])


def norms(q, k, rope, v, wq, wk, eps, pos, rows, k_out, v_out, status):
    if not len(pos):
        return q, k_out, v_out
    ang = o.angles(pos.tolist(), 1, (D, 0, 0), 10000.0, 0)
    qn, kn = (torch.tensor(o.qk_norm_rope(t.numpy(), w.numpy(), eps, ang)[0]) for t, w in ((q, wq), (k, wk)))
    for i, r in enumerate(rows.tolist()):
        if 0 <= r < k_out.shape[0]:
            k_out[r], v_out[r] = kn[i], v[i]
        elif r >= 0:
            status[0] = u.UT_ERR_INVALID_ARG
    return qn, k_out, v_out


def attention(q, k, v, cu_q, cu_k, k_len, status, left, right, sinks):
    out, lse, _ = o.window_fwd(q.numpy(), k.numpy(), v.numpy(), cu_q.numpy(), cu_k.numpy(), (left, right, sinks),
                               k_len.numpy())
    return torch.tensor(out), torch.tensor(lse)


@pytest.fixture
def setup(device, monkeypatch):
    g = torch.Generator().manual_seed(50)
    dtype, norm_dtype = torch.bfloat16, torch.float32
    if device == "cpu":
        dtype = norm_dtype = torch.float64
        monkeypatch.setattr(u, "ut_qk_norm_rope_fwd", norms)
        monkeypatch.setattr(u, "ut_window_attn_fwd", attention)

    def normal(*shape, scale=0.1):
        return (torch.randn(*shape, generator=g) * scale).to(device=device, dtype=dtype)

    w = WindowWeights(normal((H + 2 * HK) * D, C), *(torch.ones(D, dtype=norm_dtype, device=device) for _ in range(2)),
                      normal(C, H * D))
    block = WindowBlock(H, HK, D, u.rope_config(1, (D, 0, 0)), 5, 0, 2)
    return block, w, lambda n: normal(n, C, scale=1.0), lambda capacity: WindowCache(3, capacity, HK, D, dtype, device)


def prefix(counts, device):
    return torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32, device=device)


def reported(cache):
    """Whether the cache's own status word holds an error; it is cleared."""
    bad = int(cache.status.item()) == u.UT_ERR_INVALID_ARG
    cache.status.zero_()
    return bad


def near(got, want):
    if got.dtype == torch.float64:
        return not got.numel() or float((got - want).abs().max()) <= 2.0 ** -40
    return not got.numel() or err_stats(to_np(got), to_np(want))["rel_rms"] <= BF16_REL_RMS


# capacity 8: tokens a call, and the segments that have no room then
CALLS = [([7, 2, 0], []), ([1, 0, 3], []), ([1, 1, 1], [0]), ([0, 5, 1], []), ([2, 2, 3], [0, 1]), ([0, 0, 1], [2]),
         ([9, 0, 0], [0])]


@BOTH
def test_full_segments_take_nothing_and_others_stay_right(setup, device):
    block, w, tokens, cache_of = setup
    small, large = cache_of(8), cache_of(64)
    held = [0, 0, 0]
    for counts, full in CALLS:
        x = tokens(sum(counts))
        before = small.k.clone(), small.v.clone()
        got = block.extend(x, w, small, prefix(counts, device))
        assert reported(small) == bool(full), counts
        # what the others are given, without the segments that have no room
        taken = [0 if s in full else c for s, c in enumerate(counts)]
        seg = torch.repeat_interleave(torch.arange(3), torch.tensor(counts)).to(device)
        there = torch.tensor([s not in full for s in range(3)], device=device)[seg]
        want = block.extend(x[there], w, large, prefix(taken, device))
        assert not reported(large)
        assert near(got[there], want), counts
        assert torch.equal(got[~there], x[~there]), counts
        held = [a + b for a, b in zip(held, taken)]
        assert small.length.tolist() == large.length.tolist() == held
        for s in range(3):
            at, big = s * 8, s * 64
            for a, b, c in zip((small.k, small.v), before, (large.k, large.v)):
                assert near(a[at:at + held[s]], c[big:big + held[s]])
                assert torch.equal(a[at + held[s]:at + 8], b[at + held[s]:at + 8])
                if s in full:
                    assert torch.equal(a[at:at + 8], b[at:at + 8])


@BOTH
def test_a_status_word_of_the_call_is_used(setup, device):
    block, w, tokens, cache_of = setup
    cache, status = cache_of(4), torch.zeros(1, dtype=torch.int32, device=device)
    block.extend(tokens(5), w, cache, prefix([5, 0, 0], device), status=status)
    assert int(status.item()) == u.UT_ERR_INVALID_ARG and not reported(cache)
    assert cache.length.tolist() == [0, 0, 0]
    block.extend(tokens(4), w, cache, prefix([4, 0, 0], device))
    assert not reported(cache) and cache.length.tolist() == [4, 0, 0]


@BOTH
def test_places_do_not_change_the_cache(setup, device):
    cache = setup[3](8)
    cache.length.copy_(torch.tensor([3, 7, 0], dtype=torch.int32))
    pos, rows = cache.place(prefix([2, 2, 1], device), 5)
    assert pos.tolist() == [3, 4, 7, 8, 0] and cache.length.tolist() == [3, 7, 0]
    assert rows.tolist()[:2] + rows.tolist()[4:] == [3, 4, 16] and min(rows.tolist()[2:4]) >= 24

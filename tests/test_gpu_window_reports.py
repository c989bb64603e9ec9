"""Windowed attention says in the status word what is wrong with its numbers of keys, also where there is no row of keys."""
import pytest
import torch

from gpu_util import need_gpu
from test_gpu_window_attn import BOTH, i32, inputs, prefix

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def u():
    need_gpu()
    from paper_2609_23169_gb300 import ultratex
    return ultratex


@BOTH
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lq,lk,k_len,wrong", [([5], [0], [3], True), ([5], [0], [-1], True), ([5], [0], [0], False),
                                               ([4, 200], [0, 0], [0, 1], True), ([4, 200], [0, 0], [0, 0], False),
                                               ([4, 200], [0, 9], [0, 10], True), ([4, 200], [0, 9], [0, 9], False)])
def test_lengths_without_keys_are_looked_at(u, lq, lk, k_len, wrong, d, dtype):
    x = inputs(sum(lq), sum(lk), 4, 2, d, dtype)
    how = dict(left=9, sinks=2, k_len=i32(k_len))
    if len(lq) > 1:
        how.update(cu_q=i32(prefix(lq)), cu_k=i32(prefix(lk)))
    want = u.UT_ERR_INVALID_ARG if wrong else u.UT_OK
    status = u.status_word()
    out, lse = u.ut_window_attn_fwd(*x[:3], status=status, **how)
    assert int(status.item()) == want
    status = u.status_word()
    dq, dk, dv = u.ut_window_attn_bwd(*x[:3], out, lse, x[3], status=status, **how)
    assert int(status.item()) == want
    if not sum(lk):  # rows without a key, whatever k_len says
        assert not out.any() and bool(torch.isneginf(lse).all()) and not dq.any()
        assert dk.shape == dv.shape == (0, 2, d)

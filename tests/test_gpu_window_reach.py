"""How far a value that is not finite reaches in windowed attention: no farther than include/ultratex.h says.  What it
does not reach keeps its bits."""
import numpy as np
import pytest
import torch

import oracle.window_oracle as o
from gpu_util import need_gpu
from test_gpu_window_attn import BOTH, i32, inputs, prefix

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def u():
    need_gpu()
    from paper_2609_23169_gb300 import ultratex
    return ultratex


def reach(lengths, G, win, dtype, rows, keys):
    """Rows of O and dQ, and keys' gradients, that bad `keys` (of K or V) and bad `rows` (of Q or dO) may show in."""
    tile, block = (128 // G, 128) if dtype == torch.bfloat16 else (64 // G, 64)
    n = sum(lengths)
    out, dq, grad = np.zeros(n, bool), np.zeros(n, bool), np.zeros(n, bool)
    for a, b in zip(prefix(lengths), prefix(lengths)[1:]):
        on = o.seen(b - a, b - a, *win)
        bad_key = np.isin(np.arange(a, b), keys)
        bad_row = np.isin(np.arange(a, b), rows)
        for t in range(0, b - a, tile):
            if on[t:t + tile, bad_key].any():
                out[a + t:a + t + tile][:b - a - t] = True
                bad_row[t:t + tile] = True
            if not bad_row[t:t + tile].any():
                continue
            dq[a + t:a + t + tile][:b - a - t] |= bad_row[t:t + tile]
            seen = on[t:t + tile].any(0)
            for x in range(0, b - a, block):
                if seen[x:x + block].any():
                    grad[a + x:a + x + block][:b - a - x] = True
        grad[a:b] |= bad_key
        out[a:b] |= np.isin(np.arange(a, b), rows)
    return out, dq, grad


@BOTH
@pytest.mark.parametrize("heads,kv_heads,d", [(2, 2, 64), (6, 2, 64), (4, 1, 128)])
@pytest.mark.parametrize("win", [(200, 0, 0), (90, 40, 0), (150, 0, 5), (30, 10, 200)])
@pytest.mark.parametrize("where", ["v", "k", "q", "dout"])
def test_reach(u, where, win, heads, kv_heads, d, dtype):
    lengths = [700, 90, 400]
    n = sum(lengths)
    x = list(inputs(n, n, heads, kv_heads, d, dtype, seed=60))
    cu = i32(prefix(lengths))
    how = dict(left=win[0], right=win[1], sinks=win[2], cu_q=cu, cu_k=cu)

    def both():
        f = u.ut_window_attn_fwd(*x[:3], **how)
        return f, u.ut_window_attn_bwd(*x[:3], *f, x[3], **how)

    (out, lse), grads = both()
    bad = [300, 1000]
    x[("q", "k", "v", "dout").index(where)][bad] = float("nan")
    rows, keys = (bad, []) if where in ("q", "dout") else ([], bad)
    (out2, lse2), grads2 = both()
    may_out, may_dq, may_grad = reach(lengths, heads // kv_heads, win, dtype, rows, keys)
    clean_out = torch.tensor(~may_out if where != "dout" else np.ones(n, bool))
    clean_dq, clean_grad = torch.tensor(~may_dq & ~may_out), torch.tensor(~may_grad)
    assert clean_dq.any() and clean_grad.any()
    assert torch.equal(out[clean_out], out2[clean_out]) and torch.equal(lse[:, clean_out], lse2[:, clean_out])
    assert torch.equal(grads[0][clean_dq], grads2[0][clean_dq])
    for a, b in zip(grads[1:], grads2[1:]):
        assert torch.equal(a[clean_grad], b[clean_grad])
    # and what it reaches for certain: the rows that see it, or the row itself
    sees = np.zeros(n, bool)
    for a, b in zip(prefix(lengths), prefix(lengths)[1:]):
        on = o.seen(b - a, b - a, *win)
        sees[a:b] = on[:, np.isin(np.arange(a, b), keys)].any(1)
    sees[rows] = True
    assert not torch.isfinite(grads2[0].float()).flatten(1).any(1)[torch.tensor(sees)].any()

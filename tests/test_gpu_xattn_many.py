"""Cross attention with more work items than SMs: segments by the hundred, long query sides, and keys of one or of
several blocks beside one another, against the float64 oracle with the tolerances of test_gpu_xattn."""
import numpy as np
import pytest
import torch

from test_gpu_xattn import check, inputs, u  # noqa: F401

pytestmark = pytest.mark.gpu


def lengths(n, most, seed, empty=0.1):
    g = np.random.Generator(np.random.PCG64(seed))
    x = g.integers(1, most + 1, n)
    x[g.random(n) < empty] = 0
    return x.tolist()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,most_q,most_k", [(40, 300, 200), (40, 300, 90), (1100, 6, 9)])
@pytest.mark.parametrize("heads,kv_heads,d", [(8, 2, 64), (4, 2, 128)])
def test_many_segments(u, n, most_q, most_k, heads, kv_heads, d, dtype):  # noqa: F811
    lq, lk = lengths(n, most_q, n + d), lengths(n, most_k, n + d + 1)
    x = inputs(lq, lk, heads, kv_heads, d, dtype, seed=n + heads)
    mask = (torch.rand(sum(lk), generator=torch.Generator().manual_seed(n)) < 0.7).to(torch.uint8).cuda()
    check(u, *x, lq, lk)
    check(u, *x, lq, lk, mask=mask)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lq,lk", [([20011], [77]), ([20011], [300]), ([3, 15000, 40], [129, 260, 1000])])
def test_long_query_sides(u, lq, lk, d):  # noqa: F811
    """Runs of query tiles in several parts, whose dK and dV are added up at the end."""
    x = inputs(lq, lk, 3, 1, d, torch.bfloat16, seed=len(lq) + lk[0])
    check(u, *x, lq, lk, one_segment=len(lq) == 1)


def test_captured_in_a_graph(u):  # noqa: F811
    """Forward and gradient of both operators replayed from a CUDA graph repeat the calls to the bit."""
    lq, lk = [700, 1300], [300, 77]
    q, k, v, dout = inputs(lq, lk, 8, 4, 64, torch.bfloat16, seed=3)
    cu_q, cu_k = (torch.tensor(np.concatenate([[0], np.cumsum(x)]), dtype=torch.int32, device="cuda") for x in (lq, lk))
    g = torch.Generator(device="cuda").manual_seed(4)
    x, dy = (torch.randn(2000, 96, generator=g, device="cuda").bfloat16() for _ in range(2))

    def step():
        o, lse = u.ut_xattn_fwd(q, k, v, cu_q=cu_q, cu_k=cu_k)
        y, mean, rstd = u.ut_group_norm_fwd(x, None, None, 8, cu=cu_q)
        return (o, lse, *u.ut_xattn_bwd(q, k, v, o, lse, dout, cu_q=cu_q, cu_k=cu_k), y,
                *u.ut_group_norm_bwd(x, dy, None, None, mean, rstd, 8, cu=cu_q))

    want = [t.clone() for t in step()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for _ in range(3):
        for t in got:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)

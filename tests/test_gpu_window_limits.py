"""Windowed attention and the norms of queries and keys where calls meet their limits: waits that run out, rows of NaN
beside rows that count, many short segments, prefixes far out of range, calls at the same time, other devices' tensors.

Tolerances: those of the windowed attention tests, whose comparison with the float64 oracle is used."""
import pytest
import torch

from gpu_util import need_gpu, to_np
from test_gpu_window_attn import BOTH, check, i32, inputs, prefix
from test_window_host import calls

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def u():
    need_gpu()
    from paper_2609_23169_gb300 import ultratex
    return ultratex


@pytest.mark.parametrize("n,nk,d,win", [(20480, 20480, 128, (300, 300, 130)), (20480, 20480, 64, (300, 0, 4)),
                                        (5, 60000, 128, (50000, 0, 64)), (5, 60000, 64, (50000, 0, 64))])
def test_waits_are_bounded(u, n, nk, d, win, monkeypatch):
    """With no time to wait the tensor-core kernels give up, say so, and leave the device usable: several items a block,
    and keys split over blocks."""
    x = inputs(n, nk, 4, 2, d, torch.bfloat16, seed=30)
    want = u.ut_window_attn_fwd(*x[:3], *win)
    want_g = u.ut_window_attn_bwd(*x[:3], *want, x[3], *win)
    todo = (lambda s: u.ut_window_attn_fwd(*x[:3], *win, status=s),
            lambda s: u.ut_window_attn_bwd(*x[:3], *want, x[3], *win, status=s))
    monkeypatch.setenv("UT_WAIT_TIMEOUT_NS", "0")
    for f in todo:
        status = u.status_word()
        f(status)
        torch.cuda.synchronize()
        assert int(status.item()) == u.UT_ERR_TIMEOUT
    monkeypatch.delenv("UT_WAIT_TIMEOUT_NS")
    for f, ref in zip(todo, (want, want_g)):
        status = u.status_word()
        got = f(status)
        torch.cuda.synchronize()
        assert int(status.item()) == 0
        for a, b in zip(got, ref):
            assert torch.equal(a, b)


@BOTH
@pytest.mark.parametrize("win", [(30, 5, 0), (30, 0, 40), (10 ** 6, 0, 0)])
def test_keys_that_do_not_count_have_no_gradient_beside_nan(u, win, dtype):
    """A query and a dO of NaN reach the gradients of keys, but not of masked ones nor of rows behind a cache's."""
    lq, caps, k_len = [130, 20, 260], [200, 90, 300], [150, 33, 261]
    x = inputs(sum(lq), sum(caps), 4, 2, 64, dtype, seed=31)
    x[0][[3, 140, 300]] = float("nan")
    x[3][[100, 141, 150]] = float("inf")
    mask = (torch.rand(sum(caps), generator=torch.Generator().manual_seed(2)) < 0.7).to(torch.uint8)
    how = dict(left=win[0], right=win[1], sinks=win[2], cu_q=i32(prefix(lq)), cu_k=i32(prefix(caps)), k_len=i32(k_len),
               key_mask=mask.cuda())
    out, lse = u.ut_window_attn_fwd(*x[:3], **how)
    grads = u.ut_window_attn_bwd(*x[:3], out, lse, x[3], **how)
    gone = mask == 0
    for a, n, c in zip(prefix(caps), k_len, caps):
        gone[a + n:a + c] = True
    for g in grads[1:]:
        assert torch.isnan(g).any()
        assert not to_np(g)[gone.numpy()].any()


@BOTH
@pytest.mark.parametrize("heads,kv_heads,d", [(4, 2, 64), (2, 1, 128)])
def test_many_short_segments(u, heads, kv_heads, d, dtype):
    """First keys that most segments have not, of which each of many segments could have as many as there are rows."""
    lengths = [1 + (37 * i * i) % 211 for i in range(60)]
    for win in ((9, 0, 10 ** 9), (0, 20, 2 ** 31 - 1), (30, 0, 140)):
        check(u, inputs(sum(lengths), sum(lengths), heads, kv_heads, d, dtype, seed=32), lengths, lengths, win)


@pytest.mark.parametrize("rows", [64, 200])
def test_all_keys_first_keys(u, rows):
    """All keys as first keys of 2,000 segments: the bits that a window over all of them gives."""
    lengths = [rows] * 2000
    x = inputs(sum(lengths), sum(lengths), 8, 8, 64, torch.bfloat16, seed=33)
    cu = i32(prefix(lengths))

    def run(win):
        out, lse = u.ut_window_attn_fwd(*x[:3], *win, cu_q=cu, cu_k=cu)
        return out, lse, *u.ut_window_attn_bwd(*x[:3], out, lse, x[3], *win, cu_q=cu, cu_k=cu)

    for a, b in zip(run((0, 0, 10 ** 9)), run((10 ** 9, 0, 0))):
        assert torch.equal(a, b)


@BOTH
@pytest.mark.parametrize("bad", [[0, -(1 << 31), 70], [0, (1 << 31) - 1, 70], [-(1 << 31), -(1 << 31), (1 << 31) - 1],
                                 [70, 0, 0]])
def test_prefixes_far_out_of_range_are_reported(u, bad, dtype):
    x = inputs(70, 70, 2, 2, 64, dtype)
    good = i32([0, 20, 70])
    for win in ((9, 0, 2), (9, 30, 0), (0, 0, 10 ** 9)):
        for how in (dict(cu_q=i32(bad), cu_k=good), dict(cu_q=good, cu_k=i32(bad)), dict(cu_q=i32(bad), cu_k=i32(bad))):
            status = u.status_word()
            out, lse = u.ut_window_attn_fwd(*x[:3], *win, status=status, **how)
            with pytest.raises(u.UtError, match="invalid argument"):
                u.check_status(status)
            status = u.status_word()
            u.ut_window_attn_bwd(*x[:3], out, lse, x[3], *win, status=status, **how)
            with pytest.raises(u.UtError, match="invalid argument"):
                u.check_status(status)
    check(u, x, [70], [70], (9, 0, 2))


@BOTH
def test_gradients_of_two_calls_at_once(u, dtype):
    probs = [(inputs(400, 400, 4, 2, 64, dtype, seed=20), (50, 0, 3)), (inputs(30, 3000, 4, 4, 128, dtype, seed=21), (2500, 0, 9))]
    outs = [u.ut_window_attn_fwd(*x[:3], *w) for x, w in probs]
    want = [u.ut_window_attn_bwd(*x[:3], *o, x[3], *w) for (x, w), o in zip(probs, outs)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in probs]
    got = [[], []]
    for _ in range(4):
        for i, ((x, w), o) in enumerate(zip(probs, outs)):
            with torch.cuda.stream(streams[i]):
                got[i].append(u.ut_window_attn_bwd(*x[:3], *o, x[3], *w))
    torch.cuda.synchronize()
    for i in range(2):
        for g in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(g, want[i]))


def test_gradients_in_two_graphs_with_one_workspace(u):
    """Two captured backward passes that share a workspace, replayed one after the other."""
    probs = [(inputs(n, n, 4, 2, 64, torch.bfloat16, seed=n), (60, 0, 5)) for n in (700, 300)]
    outs = [u.ut_window_attn_fwd(*x[:3], *w) for x, w in probs]
    want = [u.ut_window_attn_bwd(*x[:3], *o, x[3], *w) for (x, w), o in zip(probs, outs)]
    ws = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    got, graphs = [], []
    for (x, w), o in zip(probs, outs):
        to = tuple(torch.empty_like(t) for t in (x[0], x[1], x[2]))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            u.ut_window_attn_bwd(*x[:3], *o, x[3], *w, dq=to[0], dk=to[1], dv=to[2], ws=ws)
        got.append(to)
        graphs.append(graph)
    for order in ((0, 1), (1, 0, 1)):
        for g in got:
            for t in g:
                t.zero_()
        for i in order:
            graphs[i].replay()
        torch.cuda.synchronize()
        for g, r in zip(got, want):
            assert all(torch.equal(a, b) for a, b in zip(g, r))


class NoLibrary:
    def __getattr__(self, name):
        raise AssertionError(f"{name} was called")


@pytest.mark.parametrize("i", range(4))
def test_other_devices_and_host_memory_are_refused(u, i, monkeypatch):
    norm = i == 2  # it has no workspace; the norms' gradient has no status word
    with monkeypatch.context() as m:
        m.setattr(u, "lib", NoLibrary)
        f = calls(u, "cuda")[i]
        with pytest.raises(AssertionError, match="was called"):
            f()
        with m.context() as other:
            other.setattr(torch._C, "_cuda_getDevice", lambda: 1)
            with pytest.raises(ValueError, match="current CUDA device"):
                f()
    if i != 3:
        with pytest.raises(ValueError, match="status must be"):
            f(status=torch.zeros(1, dtype=torch.int32))
    if not norm:
        with pytest.raises(ValueError, match="ws must be"):
            f(ws=torch.empty(1 << 22, dtype=torch.uint8))
        with pytest.raises(ValueError, match="ws must be"):
            f(ws=torch.empty(1 << 23, dtype=torch.uint8, device="cuda")[::2])
    f()
    torch.cuda.synchronize()


@BOTH
def test_block_without_tokens(u, dtype):
    """A block over no tokens, and caches that get none: nothing is read or written, and the gradients are zero."""
    from paper_2609_23169_gb300.window import WindowBlock, WindowCache, WindowWeights
    H, HK, D, C = 4, 2, 64, 96
    g = torch.Generator().manual_seed(40)

    def normal(*shape):
        return (torch.randn(*shape, generator=g) * 0.1).to(dtype).cuda()

    w = WindowWeights(normal((H + 2 * HK) * D, C), torch.ones(D, device="cuda"), torch.ones(D, device="cuda"), normal(C, H * D))
    block = WindowBlock(H, HK, D, u.rope_config(1, (D, 0, 0)), 10, 0, 2)
    status = u.status_word()
    x = normal(0, C)
    y = block.forward(x, w, cu=i32([0, 0, 0]), status=status)
    dx, dw = block.backward(x)
    assert y.shape == dx.shape == (0, C)
    for t, like in zip((dw.wqkv, dw.norm_q, dw.norm_k, dw.wo), (w.wqkv, w.norm_q, w.norm_k, w.wo)):
        assert t.shape == like.shape and not to_np(t).any()
    cache = WindowCache(3, 20, HK, D, dtype=dtype)
    block.extend(normal(7, C), w, cache, i32([0, 3, 3, 7]), status=status)
    before = cache.k.clone(), cache.v.clone(), cache.length.clone()
    assert before[2].tolist() == [3, 0, 4]
    assert block.extend(x, w, cache, i32([0, 0, 0, 0]), status=status).shape == (0, C)
    assert all(torch.equal(a, b) for a, b in zip(before, (cache.k, cache.v, cache.length)))
    block.extend(normal(2, C), w, cache, i32([0, 0, 2, 2]), status=status)  # one segment alone
    u.check_status(status)
    assert cache.length.tolist() == [3, 2, 4]
    rows = torch.ones(60, dtype=torch.bool, device="cuda")
    rows[20:22] = False
    assert torch.equal(cache.k[rows], before[0][rows]) and torch.equal(cache.v[rows], before[1][rows])
    assert to_np(cache.k[20:22]).any()

"""Host-side checks of the windowed-attention operators (no GPU needed): bad arguments are refused before anything is
launched, tensors off the current device too, and the key ranges of csrc/wattn.cuh against brute force."""
import ctypes
import os
import shutil
import subprocess

import pytest
import torch

INF, NAN = float("inf"), float("nan")
BOGUS = 16 * 1024  # never dereferenced: every call must fail validation first
CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_23169_gb300", "csrc")


@pytest.fixture(scope="module")
def u():
    import __graft_entry__ as g
    g.build()
    from paper_2609_23169_gb300 import ultratex
    ultratex.lib()
    return ultratex


def fill(s, f, kw):
    for n, v in {**f, **kw}.items():
        setattr(s, n, v)
    return s


def xshape(u, **kw):
    return fill(u.XattnShape(), dict(n_q=10, n_k=20, n_seg=1, n_heads=4, n_kv_heads=2, head_dim=64, dtype=u.UT_BF16,
                                     q_stride=256, k_stride=128, v_stride=128, o_stride=256, do_stride=256,
                                     dq_stride=256, dk_stride=128, dv_stride=128), kw)


def fwd(u, shape="", win="", q=BOGUS, k=BOGUS, v=BOGUS, cu_q=None, cu_k=None, k_len=None, scale=0.1, o=BOGUS, lse=BOGUS,
        ws=BOGUS, ws_bytes=1 << 40):
    shape = xshape(u) if shape == "" else shape
    win = u.Window(3, 0, 2) if win == "" else win
    return u.lib().ut_window_attn_fwd(shape and ctypes.byref(shape), win and ctypes.byref(win), q, k, v, cu_q, cu_k, k_len,
                                      None, scale, o, lse, ws, ws_bytes, None, None)


def bwd(u, shape="", win="", q=BOGUS, k_len=None, dout=BOGUS, dq=BOGUS, dk=BOGUS, dv=BOGUS, ws=BOGUS, ws_bytes=1 << 40):
    shape = xshape(u) if shape == "" else shape
    win = u.Window(3, 0, 2) if win == "" else win
    return u.lib().ut_window_attn_bwd(shape and ctypes.byref(shape), win and ctypes.byref(win), q, BOGUS, BOGUS, None,
                                      None, k_len, None, 0.1, BOGUS, BOGUS, dout, dq, dk, dv, ws, ws_bytes, None, None)


@pytest.mark.parametrize("field,value", [
    ("n_q", -1), ("n_k", -1), ("n_seg", 0), ("n_heads", 0), ("n_kv_heads", 0), ("n_kv_heads", 3), ("dtype", 7),
    ("q_stride", 248), ("k_stride", 120), ("v_stride", 132), ("o_stride", 257), ("q_stride", 1 << 60),
])
def test_attention_shapes_refused(u, field, value):
    s, w = xshape(u, **{field: value}), u.Window(3, 0, 2)
    assert fwd(u, s) == u.UT_ERR_INVALID_ARG and bwd(u, s) == u.UT_ERR_INVALID_ARG
    assert u.lib().ut_window_attn_fwd_workspace_size(ctypes.byref(s), ctypes.byref(w)) == 0
    assert u.lib().ut_window_attn_bwd_workspace_size(ctypes.byref(s), ctypes.byref(w)) == 0


@pytest.mark.parametrize("field,value", [("head_dim", 96), ("n_q", 1 << 31), ("n_k", 1 << 31), ("n_seg", 1 << 30)])
def test_attention_limits(u, field, value):
    wide = {x + "_stride": 1 << 12 for x in ("q", "k", "v", "o", "do", "dq", "dk", "dv")}
    assert fwd(u, xshape(u, **{**wide, field: value})) == u.UT_ERR_UNSUPPORTED
    assert bwd(u, xshape(u, **{**wide, field: value})) == u.UT_ERR_UNSUPPORTED


@pytest.mark.parametrize("kw", [
    dict(shape=None), dict(win=None), dict(q=None), dict(k=None), dict(v=None), dict(o=None), dict(lse=None),
    dict(q=BOGUS + 8), dict(k=BOGUS + 2), dict(v=BOGUS + 4), dict(o=BOGUS + 8), dict(lse=BOGUS + 2), dict(cu_q=BOGUS),
    dict(cu_k=BOGUS), dict(cu_q=BOGUS + 1, cu_k=BOGUS), dict(k_len=BOGUS + 2), dict(scale=0.0), dict(scale=-1.0),
    dict(scale=INF), dict(scale=NAN),
])
def test_attention_arguments_refused(u, kw):
    assert fwd(u, **kw) == u.UT_ERR_INVALID_ARG


@pytest.mark.parametrize("win", [(-1, 0, 0), (0, -1, 0), (0, 0, -1)])
def test_negative_windows_refused(u, win):
    assert fwd(u, win=u.Window(*win)) == u.UT_ERR_INVALID_ARG and bwd(u, win=u.Window(*win)) == u.UT_ERR_INVALID_ARG
    q = torch.zeros(4, 2, 64)
    with pytest.raises(ValueError):
        u.ut_window_attn_fwd(q, q, q, *win)


@pytest.mark.parametrize("kw", [dict(shape=None), dict(win=None), dict(dout=None), dict(dq=None), dict(dk=None),
                                dict(dv=None), dict(dout=BOGUS + 8), dict(dq=BOGUS + 8), dict(dk=BOGUS + 8),
                                dict(dv=BOGUS + 8), dict(q=None), dict(k_len=BOGUS + 1), dict(ws=None),
                                dict(ws=BOGUS + 4), dict(ws_bytes=8)])
def test_attention_gradient_arguments_refused(u, kw):
    assert bwd(u, **kw) == u.UT_ERR_INVALID_ARG


def test_segments_need_their_prefixes(u):
    assert fwd(u, xshape(u, n_seg=2)) == u.UT_ERR_INVALID_ARG


def test_split_keys_need_a_workspace(u):
    for dtype in (u.UT_BF16, u.UT_F32):
        s, w = xshape(u, n_q=1, n_k=100000, dtype=dtype), u.Window(1 << 20, 0, 0)
        need = u.lib().ut_window_attn_fwd_workspace_size(ctypes.byref(s), ctypes.byref(w))
        if need:  # where there are SMs for it
            assert fwd(u, s, w, ws=None) == u.UT_ERR_INVALID_ARG
            assert fwd(u, s, w, ws=BOGUS + 8) == u.UT_ERR_INVALID_ARG
            assert fwd(u, s, w, ws_bytes=need - 1) == u.UT_ERR_INVALID_ARG


def test_empty_problems_launch_nothing(u):
    assert fwd(u, xshape(u, n_q=0)) == u.UT_OK
    assert bwd(u, xshape(u, n_q=0, n_k=0)) == u.UT_OK


def nshape(u, **kw):
    return fill(u.QkNormShape(), dict(n_rows=10, n_heads=4, n_kv_heads=2, head_dim=64, dtype=u.UT_BF16, eps=1e-6,
                                      q_stride=256, k_stride=128, v_stride=128, qo_stride=256, ko_stride=128,
                                      vo_stride=128, dqo_stride=256, dko_stride=128, cache_rows=20), kw)


def nfwd(u, shape="", rope="", pos=None, q=BOGUS, k=BOGUS, v=None, wq=None, wk=None, rows=None, qo=BOGUS, ko=BOGUS, vo=None):
    shape = nshape(u) if shape == "" else shape
    rope = u.rope_config(1, (64, 0, 0)) if rope == "" else rope
    return u.lib().ut_qk_norm_rope_fwd(shape and ctypes.byref(shape), rope and ctypes.byref(rope), pos, q, k, v, wq, wk,
                                       rows, qo, ko, vo, None, None)


def nbwd(u, shape="", rope="", q=BOGUS, k=BOGUS, dqo=BOGUS, dko=BOGUS, dq=BOGUS, dk=BOGUS, dwq=None, dwk=None, ws=BOGUS,
         ws_bytes=1 << 40):
    shape = nshape(u) if shape == "" else shape
    rope = u.rope_config(1, (64, 0, 0)) if rope == "" else rope
    return u.lib().ut_qk_norm_rope_bwd(shape and ctypes.byref(shape), rope and ctypes.byref(rope), None, q, k, None, None,
                                       dqo, dko, dq, dk, dwq, dwk, ws, ws_bytes, None)


@pytest.mark.parametrize("field,value", [
    ("n_rows", -1), ("n_heads", 0), ("n_kv_heads", 0), ("head_dim", 0), ("head_dim", 128), ("dtype", 9), ("eps", 0.0),
    ("eps", -1.0), ("eps", INF), ("eps", NAN), ("q_stride", 248), ("k_stride", 132), ("qo_stride", 128), ("ko_stride", 64),
])
def test_norm_shapes_refused(u, field, value):
    s = nshape(u, **{field: value})
    assert nfwd(u, s) == u.UT_ERR_INVALID_ARG and nbwd(u, s) == u.UT_ERR_INVALID_ARG


def test_norm_limits(u):
    wide = {x: 1 << 23 for x in ("q_stride", "k_stride", "qo_stride", "ko_stride", "dqo_stride", "dko_stride")}
    assert nfwd(u, nshape(u, head_dim=32, **wide), u.rope_config(1, (32, 0, 0))) == u.UT_ERR_UNSUPPORTED
    assert nfwd(u, nshape(u, n_rows=1 << 31, **wide)) == u.UT_ERR_UNSUPPORTED
    assert nbwd(u, nshape(u, n_heads=1 << 16, **wide)) == u.UT_ERR_UNSUPPORTED


@pytest.mark.parametrize("kw", [
    dict(shape=None), dict(rope=None), dict(q=None), dict(k=None), dict(qo=None), dict(ko=None), dict(q=BOGUS + 8),
    dict(k=BOGUS + 8), dict(qo=BOGUS + 4), dict(ko=BOGUS + 4), dict(pos=BOGUS + 2), dict(wq=BOGUS + 1),
    dict(wk=BOGUS + 2), dict(rows=BOGUS + 2), dict(v=BOGUS), dict(vo=BOGUS), dict(v=BOGUS + 8, vo=BOGUS),
    dict(v=BOGUS, vo=BOGUS + 8),
])
def test_norm_arguments_refused(u, kw):
    assert nfwd(u, **kw) == u.UT_ERR_INVALID_ARG


@pytest.mark.parametrize("side,axes,theta,prefix", [(0, (64, 0, 0), 1e4, 0), (1, (62, 0, 0), 1e4, 0), (1, (63, 1, 0), 1e4, 0),
                                                    (1, (66, -2, 0), 1e4, 0), (1, (64, 0, 0), 0.0, 0),
                                                    (1, (64, 0, 0), NAN, 0), (1, (64, 0, 0), 1e4, -1)])
def test_norm_rotations_refused(u, side, axes, theta, prefix):
    rope = u.rope_config(side, axes, theta, prefix)
    assert nfwd(u, rope=rope) == u.UT_ERR_INVALID_ARG and nbwd(u, rope=rope) == u.UT_ERR_INVALID_ARG


@pytest.mark.parametrize("field", ["v_stride", "vo_stride"])
def test_norm_value_strides_refused(u, field):
    assert nfwd(u, nshape(u, **{field: 64}), v=BOGUS, vo=BOGUS) == u.UT_ERR_INVALID_ARG
    assert nfwd(u, nshape(u, cache_rows=-1), rows=BOGUS) == u.UT_ERR_INVALID_ARG


@pytest.mark.parametrize("kw", [
    dict(shape=None), dict(rope=None), dict(q=None), dict(k=None), dict(dqo=None), dict(dko=None), dict(dq=None),
    dict(dk=None), dict(dqo=BOGUS + 8), dict(dko=BOGUS + 8), dict(dq=BOGUS + 8), dict(dk=BOGUS + 8), dict(dwq=BOGUS + 2),
    dict(dwk=BOGUS + 1), dict(ws=None), dict(ws=BOGUS + 8), dict(ws_bytes=8),
])
def test_norm_gradient_arguments_refused(u, kw):
    assert nbwd(u, **kw) == u.UT_ERR_INVALID_ARG
    assert nbwd(u, nshape(u, dqo_stride=64)) == u.UT_ERR_INVALID_ARG


def test_no_rows_launch_nothing(u):
    assert nfwd(u, nshape(u, n_rows=0)) == u.UT_OK
    assert nbwd(u, nshape(u, n_rows=0), ws=None, ws_bytes=0) == u.UT_OK


class NoLibrary:
    def __getattr__(self, name):
        raise AssertionError(f"{name} was called")


def calls(u, device, dtype=torch.bfloat16):
    q = torch.zeros(8, 4, 64, dtype=dtype, device=device)
    k = torch.zeros(8, 2, 64, dtype=dtype, device=device)
    lse = torch.zeros(4, 8, device=device)
    rope = u.rope_config(1, (64, 0, 0))
    return (lambda **kw: u.ut_window_attn_fwd(q, k, k, 3, **kw),
            lambda **kw: u.ut_window_attn_bwd(q, k, k, q, lse, q, 3, **kw),
            lambda **kw: u.ut_qk_norm_rope_fwd(q, k, rope, **kw),
            lambda **kw: u.ut_qk_norm_rope_bwd(q, k, rope, q, k, **kw))


@pytest.mark.parametrize("i", range(4))
def test_cpu_tensors_are_refused(monkeypatch, i):
    from paper_2609_23169_gb300 import ultratex
    monkeypatch.setattr(ultratex, "lib", NoLibrary)
    with pytest.raises(ValueError, match="current CUDA device"):
        calls(ultratex, "cpu")[i]()
    with pytest.raises(TypeError):
        calls(ultratex, "cpu", torch.float16)[i]()


def test_binding_refusals(monkeypatch):
    from paper_2609_23169_gb300 import ultratex as u
    monkeypatch.setattr(u, "lib", NoLibrary)
    monkeypatch.setattr(u, "_current_device", lambda *a: None)  # the checks behind that one
    fwd_, bwd_, norm, norm_b = calls(u, "cpu")
    i32 = torch.int32
    for f in (fwd_, bwd_):
        with pytest.raises(ValueError, match="k_len"):
            f(k_len=torch.zeros(2, dtype=i32))
        with pytest.raises(ValueError, match="k_len"):
            f(k_len=torch.zeros(1))
        with pytest.raises(ValueError, match="key_mask"):
            f(key_mask=torch.zeros(9, dtype=torch.uint8))
        with pytest.raises(ValueError, match="both or neither"):
            f(cu_q=torch.zeros(2, dtype=i32))
    with pytest.raises(ValueError, match="lse"):
        fwd_(lse=torch.zeros(8, 4))
    with pytest.raises(ValueError, match="o must be"):
        fwd_(o=torch.zeros(8, 4, 64))
    with pytest.raises(ValueError, match="dk must be"):
        bwd_(dk=torch.zeros(8, 4, 64, dtype=torch.bfloat16))
    cache = torch.zeros(20, 2, 64, dtype=torch.bfloat16)
    for f in (norm, norm_b):
        with pytest.raises(ValueError, match="pos"):
            f(pos=torch.zeros(8, dtype=torch.int64))
        with pytest.raises(ValueError, match="wq"):
            f(wq=torch.zeros(64, dtype=torch.bfloat16))
        with pytest.raises(ValueError, match="wk"):
            f(wk=torch.zeros(32))
    with pytest.raises(ValueError, match="rows"):
        norm(rows=torch.zeros(7, dtype=i32), k_out=cache)
    with pytest.raises(ValueError, match="caches"):
        norm(rows=torch.zeros(8, dtype=i32))
    with pytest.raises(ValueError, match="caches"):
        norm(rows=torch.zeros(8, dtype=i32), k_out=cache, v=cache[:8])
    with pytest.raises(ValueError, match="k_out must be"):
        norm(k_out=cache)
    with pytest.raises(ValueError, match="v_out"):
        norm(v_out=cache[:8])
    with pytest.raises(ValueError, match="v must be"):
        norm(v=cache)
    with pytest.raises(ValueError, match="v_out must be"):
        norm(rows=torch.zeros(8, dtype=i32), k_out=cache, v=cache[:8], v_out=cache[:19])
    with pytest.raises(ValueError, match="dko must be"):
        u.ut_qk_norm_rope_bwd(torch.zeros(8, 4, 64), torch.zeros(8, 2, 64), u.rope_config(1, (64, 0, 0)),
                              torch.zeros(8, 4, 64), torch.zeros(8, 4, 64))


RANGES = r"""
#include <cstdio>
#include <vector>
#include "wattn.cuh"
using namespace ut;

static bool sees(int p, int j, int left, int right, int sinks) { return j <= p + right && (j >= p - left || j < sinks); }

// The two ranges hold exactly the keys that some token sees, their blocks each key
// of them once; the tokens of a key block are those of the definition, at least.
template <int N>
int check(int n_q, int n_k, int left, int right, int sinks, int tile) {
  int wrong = 0;
  for (int t0 = 0; t0 < n_q; t0 += tile) {
    const int t1 = t0 + tile < n_q ? t0 + tile : n_q, pa = n_k - n_q + t0, pb = n_k - n_q + t1 - 1;
    const WinRange r = win_range(pa, pb, n_k, left, right, sinks);
    std::vector<int> in(n_k, 0);
    WinBlock<N> b(r);
    for (int j = 0; j < win_blocks<N>(r); ++j, b.next(r)) {
      const int x = b.x, e = b.e;
      const WinBlock<N> same(r, j);
      wrong += same.x != x || same.e != e;
      wrong += x < 0 || e > n_k || x >= e;
      for (int key = x; key < e && key < x + N; ++key) ++in[key];
    }
    for (int key = 0; key < n_k; ++key) {
      int any = 0;
      for (int p = pa; p <= pb; ++p) any |= sees(p, key, left, right, sinks);
      wrong += in[key] > 1 || (any && !in[key]);
      // a joined range may hold keys between that nobody sees only where the ranges touch
      wrong += !any && in[key];
    }
  }
  for (int x = 0; x < n_k; x += N) {
    const int e = x + N < n_k ? x + N : n_k;
    int a, b;
    win_tokens(x, e, n_k, n_q, left, right, sinks, a, b);
    wrong += a < 0 || b > n_q || a > b;
    for (int t = 0; t < n_q; ++t) {
      int any = 0;
      for (int key = x; key < e; ++key) any |= sees(n_k - n_q + t, key, left, right, sinks);
      wrong += any && !(t >= a && t < b);
      wrong += !any && t >= a && t < b && x >= sinks;
    }
  }
  return wrong;
}

int main() {
  int wrong = 0;
  const int far = kWinMost;
  for (int n_q : {0, 1, 2, 5, 9, 17, 40})
    for (int n_k : {0, 1, 3, 8, 9, 33, 40, 41})
      for (int left : {0, 1, 6, 20, far})
        for (int right : {0, 1, 5, 30, far})
          for (int sinks : {0, 1, 4, 7, 8, 15, far})
            for (int tile : {1, 3, 8}) wrong += check<8>(n_q, n_k, left, right, sinks, tile) + check<4>(n_q, n_k, left, right, sinks, tile);
  // the largest numbers: no overflow
  const int most = kWinMost;
  const WinRange r = win_range(most - 1, most - 1, most, far, far, far), s = win_range(-most, -most + 5, 7, far, far, 3);
  wrong += r.hi != most || r.lo != 0 || s.lo != 0 || s.hi < 0 || s.hi > 7;
  int a, b;
  win_tokens(most - 1, most, most, most, far, far, 0, a, b);
  wrong += a != 0 && a != 1;
  wrong += b != most;
  win_tokens(0, 1, 1, most, far, far, 0, a, b);
  wrong += a < 0 || a > b || b > most;
  printf("%d\n", wrong);
}
"""


def test_key_ranges_against_brute_force(tmp_path):
    nvcc = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    src, exe = str(tmp_path / "host.cu"), str(tmp_path / "host")
    with open(src, "w") as f:
        f.write(RANGES)
    subprocess.run([nvcc, "-O1", "-std=c++17", "-arch=sm_103a", "-Xcompiler", "-ftrapv", "-I", CSRC, src, "-o", exe],
                   check=True)
    assert subprocess.run([exe], check=True, capture_output=True, text=True).stdout == "0\n"

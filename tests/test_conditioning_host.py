"""Host-side checks of the conditioning operators' C entry points (no GPU needed): bad arguments are refused before
anything is launched, and empty problems are no error."""
import ctypes

import pytest

INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def u():
    import __graft_entry__ as g
    g.build()
    from paper_2609_23169_gb300 import ultratex
    ultratex.lib()
    return ultratex


BOGUS = 16 * 1024  # never dereferenced: every call must fail validation first


def xshape(u, **kw):
    f = dict(n_q=10, n_k=20, n_seg=1, n_heads=4, n_kv_heads=2, head_dim=64, dtype=u.UT_BF16, q_stride=256, k_stride=128,
             v_stride=128, o_stride=256, do_stride=256, dq_stride=256, dk_stride=128, dv_stride=128)
    s = u.XattnShape()
    for n, v in {**f, **kw}.items():
        setattr(s, n, v)
    return s


def xfwd(u, shape=None, q=BOGUS, k=BOGUS, v=BOGUS, cu_q=None, cu_k=None, mask=None, scale=0.1, o=BOGUS, lse=BOGUS,
         ws=None, ws_bytes=0):
    return u.lib().ut_xattn_fwd(None if shape is None else ctypes.byref(shape), q, k, v, cu_q, cu_k, mask, scale, o,
                                lse, ws, ws_bytes, None, None)


def xbwd(u, shape=None, q=BOGUS, dout=BOGUS, dq=BOGUS, dk=BOGUS, dv=BOGUS, ws=BOGUS, ws_bytes=1 << 40, scale=0.1):
    return u.lib().ut_xattn_bwd(None if shape is None else ctypes.byref(shape), q, BOGUS, BOGUS, None, None, None,
                                scale, BOGUS, BOGUS, dout, dq, dk, dv, ws, ws_bytes, None, None)


@pytest.mark.parametrize("field,value", [
    ("n_q", -1), ("n_k", -1), ("n_seg", 0), ("n_heads", 0), ("n_kv_heads", 0), ("n_kv_heads", 3), ("dtype", 7),
    ("q_stride", 248), ("k_stride", 120), ("v_stride", 132), ("o_stride", 257), ("q_stride", 1 << 60),
])
def test_cross_attention_shapes_refused(u, field, value):
    assert xfwd(u, xshape(u, **{field: value})) == u.UT_ERR_INVALID_ARG
    assert u.lib().ut_xattn_fwd_workspace_size(ctypes.byref(xshape(u, **{field: value}))) == 0


@pytest.mark.parametrize("field,value", [("head_dim", 96), ("n_q", 1 << 31), ("n_k", 1 << 31), ("n_seg", 1 << 30)])
def test_cross_attention_limits(u, field, value):
    wide = {"q_stride": 1 << 12, "k_stride": 1 << 12, "v_stride": 1 << 12, "o_stride": 1 << 12}
    assert xfwd(u, xshape(u, **{**wide, field: value})) == u.UT_ERR_UNSUPPORTED
    many = xshape(u, n_heads=128, n_kv_heads=1, **{**wide, "q_stride": 1 << 13, "o_stride": 1 << 13})
    assert xfwd(u, many) == u.UT_ERR_UNSUPPORTED  # 128 heads of one kv head


@pytest.mark.parametrize("kw", [
    dict(shape=None), dict(q=None), dict(k=None), dict(v=None), dict(o=None), dict(lse=None), dict(q=BOGUS + 8),
    dict(k=BOGUS + 2), dict(v=BOGUS + 4), dict(o=BOGUS + 8), dict(lse=BOGUS + 2), dict(cu_q=BOGUS), dict(cu_k=BOGUS),
    dict(cu_q=BOGUS + 1, cu_k=BOGUS), dict(scale=0.0), dict(scale=-1.0), dict(scale=INF), dict(scale=NAN),
])
def test_cross_attention_arguments_refused(u, kw):
    if "shape" not in kw:
        kw["shape"] = xshape(u)
    assert xfwd(u, **kw) == u.UT_ERR_INVALID_ARG


def test_cross_attention_segments_need_their_prefixes(u):
    assert xfwd(u, xshape(u, n_seg=2)) == u.UT_ERR_INVALID_ARG


def test_cross_attention_workspace(u):
    long = xshape(u, n_q=1, n_k=100000)
    for dtype in (u.UT_BF16, u.UT_F32):
        long.dtype = dtype
        for n in ("ws", "ws_bytes"):  # keys of one query are split where there are SMs for it
            need = u.lib().ut_xattn_fwd_workspace_size(ctypes.byref(long))
            if need:
                assert xfwd(u, long, ws=BOGUS if n == "ws_bytes" else None, ws_bytes=need - 1) == u.UT_ERR_INVALID_ARG
        need = u.lib().ut_xattn_bwd_workspace_size(ctypes.byref(long))
        assert need > 0
        assert xbwd(u, long, ws=None) == u.UT_ERR_INVALID_ARG
        assert xbwd(u, long, ws=BOGUS + 4) == u.UT_ERR_INVALID_ARG
        assert xbwd(u, long, ws_bytes=need - 1) == u.UT_ERR_INVALID_ARG


@pytest.mark.parametrize("kw", [dict(shape=None), dict(dout=None), dict(dq=None), dict(dk=None), dict(dv=None),
                                dict(dout=BOGUS + 8), dict(dq=BOGUS + 8), dict(dk=BOGUS + 8), dict(dv=BOGUS + 8),
                                dict(scale=0.0), dict(q=None)])
def test_cross_attention_gradient_arguments_refused(u, kw):
    if "shape" not in kw:
        kw["shape"] = xshape(u)
    assert xbwd(u, **kw) == u.UT_ERR_INVALID_ARG


@pytest.mark.parametrize("field", ["do_stride", "dq_stride", "dk_stride", "dv_stride"])
def test_cross_attention_gradient_strides_refused(u, field):
    assert xbwd(u, xshape(u, **{field: 64})) == u.UT_ERR_INVALID_ARG


def test_empty_problems_launch_nothing(u):
    assert xfwd(u, xshape(u, n_q=0)) == u.UT_OK
    assert xbwd(u, xshape(u, n_q=0, n_k=0)) == u.UT_OK


def gshape(u, **kw):
    f = dict(n_rows=10, n_seg=1, channels=64, groups=8, dtype=u.UT_BF16, act=u.UT_ACT_SILU, eps=1e-5, x_stride=64,
             y_stride=64, dy_stride=64, dx_stride=64)
    s = u.GnormShape()
    for n, v in {**f, **kw}.items():
        setattr(s, n, v)
    return s


def gfwd(u, shape=None, x=BOGUS, cu=None, gamma=None, beta=None, y=BOGUS * 2, mean=BOGUS, rstd=BOGUS, ws=BOGUS,
         ws_bytes=1 << 40):
    return u.lib().ut_group_norm_fwd(None if shape is None else ctypes.byref(shape), x, cu, gamma, beta, y, mean, rstd,
                                     ws, ws_bytes, None, None)


def gbwd(u, shape=None, x=BOGUS, dy=BOGUS, mean=BOGUS, rstd=BOGUS, dx=BOGUS * 2, dgamma=None, dbeta=None, ws=BOGUS,
         ws_bytes=1 << 40):
    return u.lib().ut_group_norm_bwd(None if shape is None else ctypes.byref(shape), x, dy, None, None, None, mean,
                                     rstd, dx, dgamma, dbeta, ws, ws_bytes, None, None)


@pytest.mark.parametrize("field,value", [
    ("n_rows", -1), ("n_seg", 0), ("channels", 0), ("channels", 60), ("groups", 0), ("groups", 7), ("dtype", 5),
    ("act", 2), ("eps", 0.0), ("eps", -1.0), ("eps", INF), ("eps", NAN), ("x_stride", 56), ("y_stride", 68),
])
def test_group_norm_shapes_refused(u, field, value):
    assert gfwd(u, gshape(u, **{field: value})) == u.UT_ERR_INVALID_ARG
    assert u.lib().ut_group_norm_fwd_workspace_size(ctypes.byref(gshape(u, **{field: value}))) == 0


@pytest.mark.parametrize("kw", [dict(channels=8200, groups=8), dict(channels=8192, groups=8192),
                                dict(n_rows=1 << 31), dict(n_seg=1 << 30)])
def test_group_norm_limits(u, kw):
    assert gfwd(u, gshape(u, x_stride=1 << 14, y_stride=1 << 14, **kw)) == u.UT_ERR_UNSUPPORTED


@pytest.mark.parametrize("kw", [
    dict(shape=None), dict(x=None), dict(y=None), dict(mean=None), dict(rstd=None), dict(ws=None), dict(x=BOGUS + 8),
    dict(y=BOGUS + 8), dict(mean=BOGUS + 2), dict(rstd=BOGUS + 1), dict(gamma=BOGUS + 2), dict(beta=BOGUS + 2),
    dict(cu=BOGUS + 2), dict(ws=BOGUS + 8), dict(ws_bytes=8),
])
def test_group_norm_arguments_refused(u, kw):
    if "shape" not in kw:
        kw["shape"] = gshape(u)
    assert gfwd(u, **kw) == u.UT_ERR_INVALID_ARG


@pytest.mark.parametrize("kw", [
    dict(shape=None), dict(x=None), dict(dy=None), dict(dx=None), dict(mean=None), dict(rstd=None), dict(ws=None),
    dict(dy=BOGUS + 8), dict(dx=BOGUS + 8), dict(dgamma=BOGUS + 2), dict(dbeta=BOGUS + 2), dict(ws_bytes=8),
])
def test_group_norm_gradient_arguments_refused(u, kw):
    if "shape" not in kw:
        kw["shape"] = gshape(u)
    assert gbwd(u, **kw) == u.UT_ERR_INVALID_ARG

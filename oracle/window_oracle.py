"""Plain float64 numpy definitions of the windowed-attention operators (test infrastructure only).

Packed rows: segment s owns rows cu[s] .. cu[s + 1] - 1.  Nothing here is shared with the CUDA path."""
from __future__ import annotations

import numpy as np


def seen(n_q, n_k, left, right, sinks):
    """[n_q, n_k]: whether query i, at position n_k - n_q + i, sees key j."""
    p = np.arange(n_k - n_q, n_k)[:, None]
    j = np.arange(n_k)[None]
    return (j <= p + right) & ((j >= p - left) | (j < sinks))


def _segments(cu_q, cu_k, k_len, mask, win):
    for s in range(len(cu_q) - 1):
        n_q, n_k = int(cu_q[s + 1] - cu_q[s]), int(cu_k[s + 1] - cu_k[s])
        if k_len is not None:
            n_k = min(n_k, int(k_len[s]))
        on = seen(n_q, n_k, *win)
        keys = np.arange(cu_k[s], cu_k[s] + n_k)
        if mask is not None:
            on = on & (np.asarray(mask)[keys] != 0)
        yield slice(cu_q[s], cu_q[s + 1]), keys, on


def _probabilities(z, on):
    """exp(z - max) over the seen keys, its sums and LSE (rows without a key: zeros, 1 and -inf)."""
    z = np.where(on, z, -np.inf)
    m = z.max(axis=1, keepdims=True, initial=-np.inf)
    e = np.exp(z - np.where(np.isneginf(m), 0.0, m))
    total = e.sum(axis=1, keepdims=True)
    with np.errstate(divide="ignore"):
        lse = (m + np.log(total))[:, 0]
    return e / np.where(total == 0, 1.0, total), lse


def window_fwd(q, k, v, cu_q, cu_k, win, k_len=None, mask=None, scale=None):
    """(O [Nq, H, d], LSE [H, Nq], Oabs): win = (left, right, sinks); Oabs = sum_j p_j |v_j|."""
    nq, H, d = q.shape
    G = H // k.shape[1]
    scale = d ** -0.5 if scale is None else scale
    o, lse, oabs = np.zeros(q.shape), np.full((H, nq), -np.inf), np.zeros(q.shape)
    for rows, keys, on in _segments(cu_q, cu_k, k_len, mask, win):
        for h in range(H):
            p, lse[h, rows] = _probabilities(scale * (q[rows, h] @ k[keys, h // G].T), on)
            o[rows, h], oabs[rows, h] = p @ v[keys, h // G], p @ np.abs(v[keys, h // G])
    return o, lse, oabs


def window_bwd(q, k, v, dout, cu_q, cu_k, win, k_len=None, mask=None, scale=None, do_err=None):
    """dQ, dK, dV and, for each, the sum of the magnitudes of its terms: for rounding P or dS once (``*_abs``) and for
    an error of D of at most sum |dO| do_err (``*_d``; zeros without do_err [Nq, H, d])."""
    nq, H, d = q.shape
    G = H // k.shape[1]
    scale = d ** -0.5 if scale is None else scale
    r = {n: np.zeros(q.shape if n.startswith("dq") else k.shape)
         for n in ("dq", "dk", "dv", "dq_abs", "dk_abs", "dv_abs", "dq_d", "dk_d")}
    for rows, keys, on in _segments(cu_q, cu_k, k_len, mask, win):
        for h in range(H):
            g = h // G
            qs, ks, vs, do = q[rows, h], k[keys, g], v[keys, g], dout[rows, h]
            p, _ = _probabilities(scale * (qs @ ks.T), on)
            dp = do @ vs.T
            ds = p * (dp - (p * dp).sum(axis=1, keepdims=True))
            r["dq"][rows, h] = scale * (ds @ ks)
            r["dq_abs"][rows, h] = scale * (np.abs(ds) @ np.abs(ks))
            np.add.at(r["dk"][:, g], keys, scale * (ds.T @ qs))
            np.add.at(r["dk_abs"][:, g], keys, scale * (np.abs(ds).T @ np.abs(qs)))
            np.add.at(r["dv"][:, g], keys, p.T @ do)
            np.add.at(r["dv_abs"][:, g], keys, p.T @ np.abs(do))
            if do_err is not None:
                err = p * (np.abs(do) * do_err[rows, h]).sum(axis=1, keepdims=True)
                r["dq_d"][rows, h] = scale * (err @ np.abs(ks))
                np.add.at(r["dk_d"][:, g], keys, scale * (err.T @ np.abs(qs)))
    return r


def angles(pos, side, axes, theta, prefix):
    """[n, d / 2] angles of the pairs at canvas positions pos (Python integers: exact)."""
    out = []
    for t in pos:
        t = max(0, int(t) - prefix)
        at = (t // side ** 2, t % side ** 2 // side, t % side)
        out.append([at[a] * float(theta) ** (-2.0 * j / axes[a]) for a in range(3) for j in range(axes[a] // 2)])
    return np.array(out).reshape(len(pos), -1)


def _turn(x, ang):
    """The pairs of x [n, heads, d] turned by ang [n, d / 2]."""
    c, s = np.cos(ang)[:, None], np.sin(ang)[:, None]
    y = np.empty(x.shape)
    y[..., 0::2] = x[..., 0::2] * c - x[..., 1::2] * s
    y[..., 1::2] = x[..., 0::2] * s + x[..., 1::2] * c
    return y


def _pairs(x):
    """The sum of the magnitudes of each value's pair."""
    p = np.abs(x[..., 0::2]) + np.abs(x[..., 1::2])
    return np.repeat(p, 2, axis=-1)


def qk_norm_rope(x, w, eps, ang):
    """y = R(x r w) and the magnitude that its rounding errors go by."""
    r = 1.0 / np.sqrt((x * x).mean(axis=-1, keepdims=True) + eps)
    y = x * r * w
    return _turn(y, ang), _pairs(y)


def qk_norm_rope_bwd(x, w, eps, ang, dy):
    """dx, dw and the magnitudes of their terms."""
    r = 1.0 / np.sqrt((x * x).mean(axis=-1, keepdims=True) + eps)
    xh, g = x * r, _turn(dy, -ang)
    dx = r * (g * w - xh * (g * w * xh).mean(axis=-1, keepdims=True))
    ga = _pairs(dy)
    dx_abs = r * (ga * np.abs(w) + np.abs(xh) * (ga * np.abs(w * xh)).mean(axis=-1, keepdims=True))
    return dx, (g * xh).sum(axis=(0, 1)), dx_abs, (ga * np.abs(xh)).sum(axis=(0, 1))

"""Plain float64 numpy definitions of the conditioning operators (test infrastructure only).

Packed rows: segment s owns rows cu[s] .. cu[s + 1] - 1.  Nothing here is shared with the CUDA path."""
from __future__ import annotations

import numpy as np


def prefix(lengths):
    return np.concatenate([[0], np.cumsum(np.asarray(lengths, dtype=np.int64))])


def _seg_keys(cu_k, s, mask):
    keys = np.arange(cu_k[s], cu_k[s + 1])
    return keys if mask is None else keys[np.asarray(mask)[keys] != 0]


def xattn_fwd(q, k, v, cu_q, cu_k, mask=None, scale=None):
    """(O [Nq, H, d], LSE [H, Nq], Oabs): Oabs = sum_j p_j |v_j|, which bounds the effect of rounding P."""
    nq, H, d = q.shape
    G = H // k.shape[1]
    scale = d ** -0.5 if scale is None else scale
    o, lse, oabs = np.zeros(q.shape), np.full((H, nq), -np.inf), np.zeros(q.shape)
    for s in range(len(cu_q) - 1):
        keys, rows = _seg_keys(cu_k, s, mask), slice(cu_q[s], cu_q[s + 1])
        if keys.size == 0:
            continue
        for h in range(H):
            z = scale * (q[rows, h] @ k[keys, h // G].T)
            m = z.max(axis=1, keepdims=True)
            e = np.exp(z - m)
            total = e.sum(axis=1, keepdims=True)
            o[rows, h] = (e / total) @ v[keys, h // G]
            oabs[rows, h] = (e / total) @ np.abs(v[keys, h // G])
            lse[h, rows] = (m + np.log(total))[:, 0]
    return o, lse, oabs


def xattn_bwd(q, k, v, dout, cu_q, cu_k, mask=None, scale=None, do_err=None):
    """dQ, dK, dV and, for each, the sum of the magnitudes of its terms: for rounding P or dS once (``*_abs``) and
    for an error of D of at most sum |dO| do_err (``*_d``; zeros without do_err [Nq, H, d])."""
    nq, H, d = q.shape
    G = H // k.shape[1]
    scale = d ** -0.5 if scale is None else scale
    r = {n: np.zeros(q.shape if n.startswith("dq") else k.shape)
         for n in ("dq", "dk", "dv", "dq_abs", "dk_abs", "dv_abs", "dq_d", "dk_d")}
    for s in range(len(cu_q) - 1):
        keys, rows = _seg_keys(cu_k, s, mask), slice(cu_q[s], cu_q[s + 1])
        if keys.size == 0 or cu_q[s] == cu_q[s + 1]:
            continue
        for h in range(H):
            g = h // G
            qs, ks, vs, do = q[rows, h], k[keys, g], v[keys, g], dout[rows, h]
            z = scale * (qs @ ks.T)
            e = np.exp(z - z.max(axis=1, keepdims=True))
            p = e / e.sum(axis=1, keepdims=True)
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


def _act(u, act):
    return u / (1.0 + np.exp(-u)) if act else u


def group_norm_fwd(x, gamma, beta, groups, eps, act, cu):
    """(y, mean [S, G], rstd [S, G]); act: SiLU or nothing."""
    N, C = x.shape
    S, g = len(cu) - 1, groups
    y, mean, rstd = np.zeros(x.shape), np.zeros((S, g)), np.full((S, g), 1.0 / np.sqrt(eps))
    for s in range(S):
        xs = x[cu[s]:cu[s + 1]].reshape(-1, g, C // g)
        if xs.shape[0] == 0:
            continue
        mean[s] = xs.mean(axis=(0, 2))
        rstd[s] = 1.0 / np.sqrt(((xs - mean[s][None, :, None]) ** 2).mean(axis=(0, 2)) + eps)
        xh = ((xs - mean[s][None, :, None]) * rstd[s][None, :, None]).reshape(-1, C)
        y[cu[s]:cu[s + 1]] = _act(xh * gamma + beta, act)
    return y, mean, rstd


def group_norm_bwd(x, dy, gamma, beta, groups, eps, act, cu):
    """dx, dgamma, dbeta and the sums of the magnitudes of their terms (``*_abs``), which bound the effect of
    rounding: there xh = (x - mu) r counts with (|x| + |mu|) r, the magnitudes that its difference is made of, and
    act' with 1.1, its largest value (it crosses zero, where only its error is left)."""
    N, C = x.shape
    g, cpg = groups, C // groups
    _, mean, rstd = group_norm_fwd(x, gamma, beta, groups, eps, act, cu)
    r = {"dx": np.zeros(x.shape), "dx_abs": np.zeros(x.shape)}
    for n in ("dgamma", "dbeta", "dgamma_abs", "dbeta_abs"):
        r[n] = np.zeros(C)
    for s in range(len(cu) - 1):
        rows = slice(cu[s], cu[s + 1])
        n = cu[s + 1] - cu[s]
        if n == 0:
            continue
        rs = np.repeat(rstd[s], cpg)
        xh = (x[rows] - np.repeat(mean[s], cpg)) * rs
        u = xh * gamma + beta
        sig = 1.0 / (1.0 + np.exp(-u))
        du = dy[rows] * (sig * (1.0 + u * (1.0 - sig)) if act else 1.0)
        r["dbeta"] += du.sum(axis=0)
        r["dgamma"] += (du * xh).sum(axis=0)
        du_mag = 1.1 * np.abs(dy[rows])
        xh_mag = (np.abs(x[rows]) + np.abs(np.repeat(mean[s], cpg))) * rs
        r["dbeta_abs"] += du_mag.sum(axis=0)
        r["dgamma_abs"] += (du_mag * xh_mag).sum(axis=0)

        def mean_of(t):
            return np.repeat(t.reshape(n, g, cpg).mean(axis=(0, 2)), cpg)

        a, b = mean_of(gamma * du), mean_of(gamma * du * xh)
        r["dx"][rows] = rs * (gamma * du - a - xh * b)
        g_mag = np.abs(gamma) * du_mag
        r["dx_abs"][rows] = rs * (g_mag + mean_of(g_mag) + xh_mag * mean_of(g_mag * xh_mag))
    return r

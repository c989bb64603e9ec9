"""The conditioning operators: cross attention to an encoder's states and group norm with an activation, channels last.

``run`` computes them in their plain form (elementary torch operations in 32 bits, rounded once at the end) or, where
``own`` is true, through the entry points of this repository.  Both work on packed rows: the rows of all segments
(images or samples) one after another, with the prefix sums ``cu`` of the segments' lengths.
"""
import math
import random

import torch

own = False

EPS = 1e-5
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def xattn(name, n_q, n_k, segs, heads, kv_heads, d, dtype="bf16", train=False, mask=False, fused_kv=False):
    return {"name": name, "op": "xattn", "n_q": n_q, "n_k": n_k, "segs": segs, "heads": heads, "kv_heads": kv_heads,
            "d": d, "dtype": dtype, "train": train, "mask": mask, "fused_kv": fused_kv}


def gnorm(name, rows, segs, channels, groups, dtype="bf16", train=False, act="silu"):
    return {"name": name, "op": "gnorm", "rows": rows, "segs": segs, "channels": channels, "groups": groups,
            "dtype": dtype, "train": train, "act": act}


def listed():
    return [
        # one learned query for each of four samples over a short prompt, shared kv heads: what counts is latency
        xattn("xattn single token", 4, 231, 4, 24, 8, 64, mask=True),
        # one pooling query over all retained tokens of a 2048 canvas: the keys are the long axis
        xattn("xattn pooling query", 1, 85202, 1, 24, 24, 128, fused_kv=True),
        # retained tokens of a 1024 canvas, each image against its own padded image-encoder states
        xattn("xattn per image", 23959, 13 * 257, 13, 24, 24, 64, mask=True, fused_kv=True),
        # all retained tokens of a 2048 canvas against the 512 text tokens
        xattn("xattn text 2048", 85202, 512, 1, 24, 24, 128),
        # training step of a ragged batch against short padded prompts, shared kv heads
        xattn("xattn train prompts", 7780, 13 * 77, 13, 24, 8, 64, train=True, mask=True),
        # training step of a 1024 canvas against the 512 text tokens
        xattn("xattn train text 1024", 23959, 512, 1, 24, 24, 128, train=True, fused_kv=True),
        # the 32-bit configuration, as it serves to check a model's training
        xattn("xattn train f32", 2501, 301, 3, 8, 4, 64, dtype="f32", train=True, mask=True),
        # one image's 16 x 16 feature map: latency
        gnorm("gnorm small map", 256, 1, 320, 32),
        # decoder features of six views at 256 x 256
        gnorm("gnorm decoder 256", 6 * 65536, 6, 512, 32),
        # full-resolution decoder features of one 2048 image, in front of the output layer
        gnorm("gnorm decoder 2048", 2048 * 2048, 1, 128, 32),
        # training step on the retained tokens of a 2048 canvas, image by image
        gnorm("gnorm train canvas", 85202, 13, 640, 32, train=True),
        # 32 bits, no activation, few rows for each sample
        gnorm("gnorm train f32", 7780, 13, 96, 8, dtype="f32", train=True, act="none"),
    ]


def log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    train = rng.random() < 0.5
    segs = rng.choice([1, 1, 2, 6, 13, 24])
    if rng.random() < 0.5:
        d = rng.choice([64, 128])
        kv_heads = rng.choice([1, 2, 4, 8, 24])
        heads = kv_heads * rng.choice([g for g in (1, 2, 3, 4, 8) if g * kv_heads <= 24])
        if not train and rng.random() < 0.4:  # few queries over long states
            n_q, n_k = segs * log_uniform(rng, 1, 24), segs * log_uniform(rng, 60, 85202 // segs)
        else:
            n_q, n_k = log_uniform(rng, 40 * segs, 85202), segs * log_uniform(rng, 9, 1031)
        most = 85202 * 512 * 24 * 128 // (24 if dtype == "f32" else 4 if train else 1)
        n_q = max(segs, min(n_q, most * segs // (n_k * heads * d)))
        case = xattn("", n_q, n_k, segs, heads, kv_heads, d, dtype, train, rng.random() < 0.5, rng.random() < 0.5)
    else:
        groups = rng.choice([1, 4, 8, 32])
        channels = max(groups, 8) * rng.choice([1, 2, 3, 5, 8, 12, 16, 20])
        most = 2048 * 2048 * 128 // (4 if train else 2 if dtype == "f32" else 1)
        rows = min(log_uniform(rng, 16 * segs, 1 << 21), most // channels)
        case = gnorm("", rows, segs, channels, groups, dtype, train, rng.choice(["silu", "silu", "none"]))
    del case["name"]
    return case


def lengths(total, n, holes):
    """The lengths of n ragged segments of `total` rows; with holes, the second of eight or more has none."""
    rng = random.Random(1009 * total + n)
    w = [0.3 + 1.4 * rng.random() for _ in range(n)]
    if holes and n >= 8:
        w[1] = 0.0
    ls = [int(total * x / sum(w)) for x in w]
    ls[-1] += total - sum(ls)
    return ls


def prefix(ls):
    at = [0]
    for x in ls:
        at.append(at[-1] + x)
    return at


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(seed)
    dt = DTYPES[case["dtype"]]

    def normal(*shape, scale=1.0):
        return torch.empty(shape, dtype=dt, device=dev).normal_(0.0, scale, generator=gen)

    st = dict(case)
    n = case["segs"]
    if case["op"] == "xattn":
        H, Hk, d, nq, nk = (case[x] for x in ("heads", "kv_heads", "d", "n_q", "n_k"))
        lq, lk = lengths(nq, n, False), lengths(nk, n, True)
        st["q"] = normal(nq, H, d, scale=1.3)
        if case["fused_kv"]:  # K and V as the two halves of one projection's rows
            kv = normal(nk, 2, Hk, d)
            st["k"], st["v"] = kv[:, 0], kv[:, 1]
        else:
            st["k"], st["v"] = normal(nk, Hk, d), normal(nk, Hk, d)
        st["cu_q"] = torch.tensor(prefix(lq), dtype=torch.int32, device=dev) if n > 1 else None
        st["cu_k"] = torch.tensor(prefix(lk), dtype=torch.int32, device=dev) if n > 1 else None
        st["max_q"], st["max_k"] = max(lq), max(lk)
        st["key_mask"] = None
        if case["mask"]:
            keep = torch.rand(nk, device=dev, generator=gen) < 0.8
            if n > 2:  # a sample without a prompt
                keep[prefix(lk)[2]:prefix(lk)[3]] = False
            st["key_mask"] = keep.to(torch.uint8)
        if case["train"]:
            st["dout"] = normal(nq, H, d)
        return st
    C, N = case["channels"], case["rows"]
    ls = lengths(N, n, False)
    shift = torch.empty(C, dtype=torch.float32, device=dev).normal_(0.5, 0.5, generator=gen)
    st["x"] = normal(N, C, scale=1.5).add_(shift.to(dt))
    st["gamma"] = torch.empty(C, dtype=torch.float32, device=dev).normal_(1.0, 0.2, generator=gen)
    st["beta"] = torch.empty(C, dtype=torch.float32, device=dev).normal_(0.0, 0.3, generator=gen)
    st["cu"] = torch.tensor(prefix(ls), dtype=torch.int32, device=dev) if n > 1 else None
    st["max_rows"] = max(ls)
    if case["train"]:
        st["dy"] = normal(N, C)
    return st


def padded(cu, n, most, dev):
    """Row indexes [segments, most] of the segments, which of them exist, and each row's segment and place."""
    if cu is None:
        cu = torch.tensor([0, n], dtype=torch.int32, device=dev)
    at = torch.arange(most, device=dev)
    length = (cu[1:] - cu[:-1]).long()
    rows = (cu[:-1, None] + at).clamp(max=max(n - 1, 0)).long()
    row = torch.arange(n, device=dev)
    seg = torch.bucketize(row, cu[1:].long(), right=True)
    return rows, at < length[:, None], length, seg, row - cu[:-1].long()[seg]


def plain_xattn(st):
    q, k, v = st["q"].float(), st["k"].float(), st["v"].float()
    dt, dev = st["q"].dtype, q.device
    (nq, H, d), (nk, Hk) = q.shape, k.shape[:2]
    G, scale = H // Hk, d ** -0.5
    rq, real, _, seg, place = padded(st["cu_q"], nq, st["max_q"], dev)
    rk, there, _, kseg, kplace = padded(st["cu_k"], nk, st["max_k"], dev)
    B, mq, mk = rq.shape[0], rq.shape[1], rk.shape[1]
    if st["key_mask"] is not None:
        there = there & (st["key_mask"][rk] != 0)

    def heads_first(x):  # [rows, H, d] -> [B, Hk, G * mq, d]: the heads that share a kv head are rows of one product
        return torch.where(real[:, :, None, None], x[rq], 0.0).view(B, mq, Hk, G, d).permute(0, 2, 3, 1, 4).reshape(B, Hk, G * mq, d)

    def packed(x):  # and back
        return x.view(B, Hk, G, mq, -1).permute(0, 3, 1, 2, 4).reshape(B, mq, H, -1)[seg, place]

    qp, kp, vp = heads_first(q), k[rk].permute(0, 2, 1, 3), v[rk].permute(0, 2, 1, 3)
    s = (qp @ kp.transpose(2, 3)) * scale
    s = s.masked_fill(~there[:, None, None, :], -math.inf)
    m = s.amax(3, keepdim=True)
    p = torch.exp(s - torch.where(m == -math.inf, 0.0, m))
    del s
    total = p.sum(3, keepdim=True)
    p = p / torch.where(total == 0, 1.0, total)
    o = p @ vp
    lse = packed(m + torch.log(total))[..., 0].t()
    out = [packed(o).to(dt), lse]
    if st["train"]:
        do = heads_first(st["dout"].float())
        dv = p.transpose(2, 3) @ do
        ds = p * (do @ vp.transpose(2, 3) - (do * o).sum(3, keepdim=True))
        dq = (ds @ kp) * scale
        dk = (ds.transpose(2, 3) @ qp) * scale
        out += [packed(dq).to(dt)] + [x.permute(0, 2, 1, 3)[kseg, kplace].to(dt) for x in (dk, dv)]
    return out


def plain_gnorm(st):
    x, gamma, beta, G = st["x"].float(), st["gamma"], st["beta"], st["groups"]
    dt, (N, C) = st["x"].dtype, x.shape
    rows, there, length, seg, place = padded(st["cu"], N, st["max_rows"], x.device)
    B, mx = rows.shape
    there = there[:, :, None, None]

    def grouped(t):
        return torch.where(there, t[rows].view(B, mx, G, C // G), 0.0)

    def packed(t):
        return t.view(B, mx, C)[seg, place]

    g, b = gamma.view(G, C // G), beta.view(G, C // G)
    count = (length * (C // G)).clamp(min=1).float().view(B, 1, 1, 1)
    xg = grouped(x)
    mean = xg.sum((1, 3), keepdim=True) / count
    xg = torch.where(there, xg - mean, 0.0)
    rstd = 1.0 / torch.sqrt((xg * xg).sum((1, 3), keepdim=True) / count + EPS)
    xh = xg * rstd
    u = xh * g + b
    sig = 1.0 / (1.0 + torch.exp(-u)) if st["act"] == "silu" else None
    y = u * sig if st["act"] == "silu" else u
    out = [packed(y).to(dt), mean.view(B, G), rstd.view(B, G)]
    if st["train"]:
        du = grouped(st["dy"].float())
        if st["act"] == "silu":
            du = du * (sig * (1.0 + u * (1.0 - sig)))
        dbeta, dgamma = du.sum((0, 1)).view(C), (du * xh).sum((0, 1)).view(C)
        dg = du * g
        a, c = dg.sum((1, 3), keepdim=True) / count, (dg * xh).sum((1, 3), keepdim=True) / count
        out += [packed(rstd * (dg - a - xh * c)).to(dt), dgamma, dbeta]
    return out


def run(st):
    if not own:
        return plain_xattn(st) if st["op"] == "xattn" else plain_gnorm(st)
    from paper_2609_23169_gb300 import ultratex as u
    if st["op"] == "xattn":
        how = {"cu_q": st["cu_q"], "cu_k": st["cu_k"], "key_mask": st["key_mask"]}
        o, lse = u.ut_xattn_fwd(st["q"], st["k"], st["v"], **how)
        if not st["train"]:
            return [o, lse]
        return [o, lse, *u.ut_xattn_bwd(st["q"], st["k"], st["v"], o, lse, st["dout"], **how)]
    act = u.UT_ACT_SILU if st["act"] == "silu" else u.UT_ACT_NONE
    how = {"eps": EPS, "act": act, "cu": st["cu"]}
    y, mean, rstd = u.ut_group_norm_fwd(st["x"], st["gamma"], st["beta"], st["groups"], **how)
    if not st["train"]:
        return [y, mean, rstd]
    del how["eps"]
    return [y, mean, rstd, *u.ut_group_norm_bwd(st["x"], st["dy"], st["gamma"], st["beta"], mean, rstd, st["groups"],
                                                **how)]


def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "xattn":
        H, Hk, d, nq, nk, n = (case[x] for x in ("heads", "kv_heads", "d", "n_q", "n_k", "segs"))
        lq, lk = lengths(nq, n, False), lengths(nk, n, True)
        if case["mask"] and n > 2:
            lk[2] = 0
        pairs = sum(a * b for a, b in zip(lq, lk)) * (0.8 if case["mask"] else 1.0)  # four of five keys are kept
        qo, kv = nq * H * d * e, 2 * nk * Hk * d * e
        small = 4 * nq * H + 8 * (n + 1) + (nk if case["mask"] else 0)
        if case["train"]:
            return {"bytes": 4 * qo + 2 * kv + small, "flops": 14 * H * d * pairs}
        return {"bytes": 2 * qo + kv + small, "flops": 4 * H * d * pairs}
    N, C, n = case["rows"], case["channels"], case["segs"]
    small = 8 * C + 8 * n * case["groups"] + 4 * (n + 1)
    if case["train"]:
        return {"bytes": 4 * N * C * e + small + 8 * C, "flops": 30 * N * C}
    return {"bytes": 2 * N * C * e + small, "flops": 12 * N * C}


def exact(case, seed):
    st = prepare(case, seed)
    n = case["segs"]
    if case["op"] == "xattn":
        H, Hk, d, nq, nk = (case[x] for x in ("heads", "kv_heads", "d", "n_q", "n_k"))
        aq, ak = prefix(lengths(nq, n, False)), prefix(lengths(nk, n, True))
        dev = st["q"].device
        z = dict(dtype=torch.float64, device=dev)
        out = [torch.zeros(nq, H, d, **z), torch.full((H, nq), -math.inf, **z)]
        if case["train"]:
            out += [torch.zeros(nq, H, d, **z), torch.zeros(nk, Hk, d, **z), torch.zeros(nk, Hk, d, **z)]
        for s in range(n):
            keys = torch.arange(ak[s], ak[s + 1], device=dev)
            if st["key_mask"] is not None:
                keys = keys[st["key_mask"][keys] != 0]
            if aq[s] == aq[s + 1] or keys.numel() == 0:
                continue
            mine = slice(aq[s], aq[s + 1])
            for h in range(H):
                kh = h * Hk // H
                q, k, v = st["q"][mine, h].double(), st["k"][keys, kh].double(), st["v"][keys, kh].double()
                for t in (q, k, v):
                    t.requires_grad_(case["train"])
                s_ = torch.einsum("id,jd->ij", q, k) / math.sqrt(d)
                o = torch.einsum("ij,jd->id", torch.softmax(s_, 1), v)
                out[0][mine, h], out[1][h, mine] = o.detach(), torch.logsumexp(s_.detach(), 1)
                if case["train"]:
                    gq, gk, gv = torch.autograd.grad(o, (q, k, v), st["dout"][mine, h].double())
                    out[2][mine, h] = gq
                    out[3][:, kh].index_add_(0, keys, gk)
                    out[4][:, kh].index_add_(0, keys, gv)
        return out
    G, C, N = case["groups"], case["channels"], case["rows"]
    at = prefix(lengths(N, n, False))
    gamma, beta = (st[t].double().requires_grad_(case["train"]) for t in ("gamma", "beta"))
    ys, means, rstds, dxs, dg, db = [], [], [], [], torch.zeros_like(gamma), torch.zeros_like(beta)
    for s in range(n):
        x = st["x"][at[s]:at[s + 1]].double().requires_grad_(case["train"])
        x3 = x.view(-1, G, C // G)
        var, mean = torch.var_mean(x3, (0, 2), correction=0, keepdim=True)
        rstd = (var + EPS).rsqrt()
        u = ((x3 - mean) * rstd).reshape(-1, C) * gamma + beta
        y = torch.nn.functional.silu(u) if case["act"] == "silu" else u
        ys.append(y.detach())
        means.append(mean.detach().view(1, G))
        rstds.append(rstd.detach().view(1, G))
        if case["train"]:
            gx, gg, gb = torch.autograd.grad(y, (x, gamma, beta), st["dy"][at[s]:at[s + 1]].double())
            dxs.append(gx)
            dg, db = dg + gg, db + gb
    out = [torch.cat(ys), torch.cat(means), torch.cat(rstds)]
    return out + [torch.cat(dxs), dg.detach(), db.detach()] if case["train"] else out

"""The windowed-attention operators: norms of queries and keys with the position rotation, and attention with a sliding
window and first tokens that stay visible.

``run`` computes them in their plain form (elementary torch operations in 32 bits, angles in 64, rounded once at the end)
or, where ``own`` is true, through the entry points of this repository.  Both work on packed rows; the attention's are the
rows of all segments (images or samples) one after another, with the prefix sums ``cu`` of the segments' lengths.
"""
import math
import random

import numpy as np
import torch

own = False

EPS = 1e-6
THETA = 10000.0
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIDE = 128  # tokens per side of a 2048 image; 13 images a canvas, after 512 text tokens
IMAGES, TEXT = 13, 512


def qknorm(name, rows, heads, kv_heads, d, dtype="bf16", train=False, pos="canvas", cap=0):
    """Queries and keys as slices of one projection's rows.  cap: keys and values go to rows of a cache of so many."""
    return {"name": name, "op": "qknorm", "rows": rows, "heads": heads, "kv_heads": kv_heads, "d": d, "dtype": dtype,
            "train": train, "pos": pos, "cap": cap}


def window(name, n_q, segs, heads, kv_heads, d, left, right, sinks, dtype="bf16", train=False, mask=False, cap=0):
    """cap: each segment's keys are the filled rows of a cache of so many, its queries their last; else its own rows."""
    return {"name": name, "op": "window", "n_q": n_q, "segs": segs, "heads": heads, "kv_heads": kv_heads, "d": d,
            "left": left, "right": right, "sinks": sinks, "dtype": dtype, "train": train, "mask": mask, "cap": cap}


def listed():
    return [
        # one new token of each of four samples, its key and value put into their caches: what counts is latency
        qknorm("qknorm single tokens", 4, 24, 8, 64, pos="line", cap=4 * 4096),
        # a ragged prompt on its way into the cache
        qknorm("qknorm prompt", 7781, 24, 8, 64, pos="line", cap=8192),
        # all retained tokens of a 2048 canvas behind its 512 text tokens
        qknorm("qknorm canvas 2048", 85714, 24, 24, 128),
        # training step on the retained tokens of a 1024 canvas
        qknorm("qknorm train 1024", 23959, 24, 24, 128, train=True),
        # the 32-bit configuration, as it serves to check a model's training
        qknorm("qknorm train f32", 2501, 8, 4, 64, dtype="f32", train=True, pos="line"),
        # one new token of each of four samples over their caches, shared kv heads
        window("window single tokens", 4, 4, 24, 8, 64, 1023, 0, 4, cap=4096),
        # a few new tokens over a long cache: the keys are the long axis
        window("window long cache", 13, 1, 24, 24, 128, 40000, 0, 512, cap=85714),
        # all retained tokens of a 2048 canvas, each among its neighbours and the 512 text tokens
        window("window canvas 2048", 85714, 1, 24, 24, 128, 512, 512, 512),
        # retained tokens of a 1024 canvas image by image, some of them masked
        window("window per image", 23959, 13, 24, 24, 64, 192, 192, 0, mask=True),
        # training step of a 1024 canvas behind its text tokens
        window("window train 1024", 24471, 1, 24, 24, 128, 512, 512, 512, train=True),
        # causal training step on a ragged padded batch, shared kv heads
        window("window train causal", 7780, 13, 24, 8, 64, 255, 0, 4, train=True, mask=True),
        # the 32-bit configuration
        window("window train f32", 2501, 3, 8, 4, 64, 100, 28, 7, dtype="f32", train=True, mask=True),
    ]


def log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    train = rng.random() < 0.5
    d = rng.choice([64, 128])
    kv_heads = rng.choice([1, 2, 4, 8, 24])
    heads = kv_heads * rng.choice([g for g in (1, 2, 3, 4, 8) if g * kv_heads <= 24])
    if rng.random() < 0.4:
        cap = 0 if train else rng.choice([0, 1])
        rows = log_uniform(rng, 1, 85714)
        rows = min(rows, 85714 * 24 * 128 // ((heads + kv_heads) * d * (3 if train else 1) * (2 if dtype == "f32" else 1)))
        case = qknorm("", max(1, rows), heads, kv_heads, d, dtype, train, rng.choice(["canvas", "line"]),
                      cap * (rows + log_uniform(rng, 1, 20000)))
    else:
        segs = rng.choice([1, 1, 2, 6, 13, 24])
        sinks = rng.choice([0, 1, 4, 77, 512])
        right = rng.choice([0, 1]) * log_uniform(rng, 1, 600)
        most = 85714 * 1537 * 24 * 128 // (24 if dtype == "f32" else 4 if train else 1)
        if not train and rng.random() < 0.4:  # new tokens over caches
            n_q = segs * log_uniform(rng, 1, 24)
            cap = log_uniform(rng, max(60, n_q // segs), 85714 // segs)
            left = log_uniform(rng, 16, 40000)
        else:
            cap, left = 0, log_uniform(rng, 100, 1500)
            n_q = log_uniform(rng, 40 * segs, 85714)
            n_q = max(segs, min(n_q, most // ((left + right + sinks + 512) * heads * 128)))
        case = window("", n_q, segs, heads, kv_heads, d, left, right, sinks, dtype, train, rng.random() < 0.4, cap)
    del case["name"]
    return case


def lengths(total, n):
    """The lengths of n ragged segments of `total` rows; of eight or more the second has none."""
    rng = random.Random(1009 * total + n)
    w = [0.3 + 1.4 * rng.random() for _ in range(n)]
    if n >= 8:
        w[1] = 0.0
    ls = [int(total * x / sum(w)) for x in w]
    ls[-1] += total - sum(ls)
    return ls


def key_lengths(case):
    """Queries and keys of every segment."""
    n, cap = case["segs"], case["cap"]
    if not cap:
        ls = lengths(case["n_q"], n)
        return ls, ls
    lq = [case["n_q"] // n] * n
    lq[0] += case["n_q"] - sum(lq)
    rng = random.Random(2003 * cap + n)
    return lq, [cap if s == 0 else max(lq[s], int(cap * (0.4 + 0.6 * rng.random()))) for s in range(n)]


def prefix(ls):
    at = [0]
    for x in ls:
        at.append(at[-1] + x)
    return at


def axes(d):
    """How a canvas splits a head's dimensions over image, y and x."""
    return (d // 8, (d - d // 8) // 2, (d - d // 8) // 2)


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(seed)
    dt = DTYPES[case["dtype"]]

    def normal(*shape, scale=1.0, mean=0.0, dtype=dt):
        return torch.empty(shape, dtype=dtype, device=dev).normal_(mean, scale, generator=gen)

    st = dict(case)
    H, Hk, d = case["heads"], case["kv_heads"], case["d"]
    if case["op"] == "qknorm":
        n, st["kind"] = case["rows"], case["pos"]
        qkv = normal(n, H + 2 * Hk, d, scale=1.5)
        st["q"], st["k"], st["v"] = qkv[:, :H], qkv[:, H:H + Hk], qkv[:, H + Hk:]
        st["wq"], st["wk"] = (normal(d, mean=1.0, scale=0.2, dtype=torch.float32) for _ in range(2))
        if case["pos"] == "canvas":  # ascending canvas positions, the text tokens first
            at = torch.rand(n, device=dev, generator=gen).sort().values * (TEXT + IMAGES * SIDE * SIDE)
            st["pos"] = at.int()
        else:  # positions of a long text, each sample's from its own start
            start = torch.randint(0, 131072, (1,), device=dev, generator=gen)
            st["pos"] = (start + torch.arange(n, device=dev) * (7919 if n < 64 else 1)).int()
        if case["cap"]:  # distinct rows of the cache
            st["at"] = torch.randperm(case["cap"], device=dev, generator=gen)[:n].int()
            st["k_cache"], st["v_cache"] = normal(case["cap"], Hk, d), normal(case["cap"], Hk, d)
        if case["train"]:
            st["dqo"], st["dko"] = normal(n, H, d), normal(n, Hk, d)
        return st
    lq, lk = key_lengths(case)
    n, segs, cap = case["n_q"], case["segs"], case["cap"]
    if cap:
        nk = segs * cap
        st["q"], st["k"], st["v"] = normal(n, H, d, scale=1.3), normal(nk, Hk, d), normal(nk, Hk, d)
        st["cu_k"] = torch.arange(segs + 1, dtype=torch.int32, device=dev) * cap
        st["k_len"] = torch.tensor(lk, dtype=torch.int32, device=dev)
    else:
        nk = n
        qkv = normal(n, H + 2 * Hk, d, scale=1.1)
        st["q"], st["k"], st["v"] = qkv[:, :H], qkv[:, H:H + Hk], qkv[:, H + Hk:]
        st["k_len"] = None
    st["cu_q"] = torch.tensor(prefix(lq), dtype=torch.int32, device=dev)
    if not cap:
        st["cu_k"] = st["cu_q"]
    if segs == 1:
        st["cu_q"] = st["cu_k"] = None
    st["max_q"], st["max_k"] = max(lq), max(lk)
    st["key_mask"] = (torch.rand(nk, device=dev, generator=gen) < 0.9).to(torch.uint8) if case["mask"] else None
    if case["train"]:
        st["dout"] = normal(n, H, d)
    return st


def plain_angles(st):
    """Angles [rows, d / 2] of the pairs, in 64 bits."""
    d, pos = st["d"], st["pos"].double()
    if st["kind"] == "line":
        return pos[:, None] * THETA ** (-2.0 * torch.arange(d // 2, device=pos.device).double() / d)
    t = (pos - TEXT).clamp(min=0)
    image, y, x = torch.floor(t / SIDE ** 2), torch.floor(t / SIDE) % SIDE, t % SIDE
    parts = [c[:, None] * THETA ** (-2.0 * torch.arange(a // 2, device=pos.device).double() / a)
             for c, a in zip((image, y, x), axes(d))]
    return torch.cat(parts, 1)


def plain_qknorm(st):
    dt, n, d = st["q"].dtype, st["rows"], st["d"]
    ang = plain_angles(st)
    cos, sin = torch.cos(ang).float()[:, None, :], torch.sin(ang).float()[:, None, :]

    def forward(x, w):
        x = x.float()
        r = 1.0 / torch.sqrt((x * x).sum(2, keepdim=True) / d + EPS)
        y = (x * r * w).view(n, -1, d // 2, 2)
        a, b = y[..., 0], y[..., 1]
        return torch.stack((a * cos - b * sin, a * sin + b * cos), 3).view(n, -1, d).to(dt)

    def backward(x, w, dy):
        x, g = x.float(), dy.float().view(n, -1, d // 2, 2)
        a, b = g[..., 0], g[..., 1]
        g = torch.stack((a * cos + b * sin, b * cos - a * sin), 3).view(n, -1, d)
        r = 1.0 / torch.sqrt((x * x).sum(2, keepdim=True) / d + EPS)
        xh = x * r
        dw = (g * xh).sum((0, 1))
        g = g * w
        return (r * (g - xh * ((g * xh).sum(2, keepdim=True) / d))).to(dt), dw

    qo, ko = forward(st["q"], st["wq"]), forward(st["k"], st["wk"])
    if st["cap"]:
        at = st["at"].long()
        st["k_cache"][at] = ko
        st["v_cache"][at] = st["v"]
        return [qo, st["k_cache"], st["v_cache"]]
    if not st["train"]:
        return [qo, ko]
    (dq, dwq), (dk, dwk) = backward(st["q"], st["wq"], st["dqo"]), backward(st["k"], st["wk"], st["dko"])
    return [qo, ko, dq, dk, dwq, dwk]


def plain_window(st):
    """Rows in blocks of C, each against the first keys and the keys around it, all blocks of all segments at once."""
    q, k, v = st["q"].float(), st["k"].float(), st["v"].float()
    dt, dev = st["q"].dtype, q.device
    (nq, H, d), (nk, Hk) = q.shape, k.shape[:2]
    G, scale = H // Hk, d ** -0.5
    left, right, sinks = (min(st[x], st["max_k"]) for x in ("left", "right", "sinks"))
    cu_q = st["cu_q"].long() if st["cu_q"] is not None else torch.tensor([0, nq], device=dev)
    cu_k = st["cu_k"].long() if st["cu_k"] is not None else torch.tensor([0, nk], device=dev)
    lq = cu_q[1:] - cu_q[:-1]
    lk = cu_k[1:] - cu_k[:-1] if st["k_len"] is None else st["k_len"].long()
    B, C = lq.numel(), min(st["max_q"], 512)
    nb = -(-st["max_q"] // C)
    place = torch.arange(nb * C, device=dev).view(nb, C)
    real = place < lq[:, None, None]                                     # [B, nb, C]
    rq = (cu_q[:-1, None, None] + place).clamp(max=nq - 1)
    p = (lk - lq)[:, None, None] + place
    near = p[:, :, :1] - left + torch.arange(C + left + right, device=dev)
    first = torch.arange(sinks, device=dev).expand(B, nb, sinks)
    key = torch.cat((first, near), 2)                                    # [B, nb, K]
    there = (key >= 0) & (key < lk[:, None, None])
    there[:, :, sinks:] &= near >= sinks
    rk = (cu_k[:-1, None, None] + key).clamp(0, nk - 1)
    if st["key_mask"] is not None:
        there = there & (st["key_mask"][rk] != 0)
    low = (p - left)[..., None].expand(B, nb, C, key.shape[2])
    low = torch.where(torch.arange(key.shape[2], device=dev) < sinks, 0, low)
    seen = there[:, :, None] & (key[:, :, None] >= low) & (key[:, :, None] <= (p + right)[..., None])
    seen = seen[:, :, None, None]                                        # [B, nb, 1, 1, C, K]

    def rows_of(x):  # [rows, H, d] -> [B, nb, Hk, G * C, d]: the heads that share a kv head are rows of one product
        x = torch.where(real[..., None, None], x[rq], 0.0)
        return x.view(B, nb, C, Hk, G, d).permute(0, 1, 3, 4, 2, 5).reshape(B, nb, Hk, G * C, d)

    def keys_of(x):  # [rows, Hk, d] -> [B, nb, Hk, K, d]
        return torch.where(there[..., None, None], x[rk], 0.0).permute(0, 1, 3, 2, 4)

    seg = torch.bucketize(torch.arange(nq, device=dev), cu_q[1:], right=True)
    back = seg * (nb * C) + torch.arange(nq, device=dev) - cu_q[seg]

    def packed(x):
        return x.view(B, nb, Hk, G, C, -1).permute(0, 1, 4, 2, 3, 5).reshape(B * nb * C, H, -1)[back]

    qp, kp, vp = rows_of(q), keys_of(k), keys_of(v)
    s = (qp @ kp.transpose(3, 4)) * scale
    s = s.view(B, nb, Hk, G, C, -1).masked_fill(~seen, -math.inf).view(B, nb, Hk, G * C, -1)
    m = s.amax(4, keepdim=True)
    pr = torch.exp(s - torch.where(m == -math.inf, 0.0, m))
    del s
    total = pr.sum(4, keepdim=True)
    pr = pr / torch.where(total == 0, 1.0, total)
    o = pr @ vp
    out = [packed(o).to(dt), packed(m + torch.log(total))[..., 0].t().contiguous()]
    if st["train"]:
        do = rows_of(st["dout"].float())
        ds = pr * (do @ vp.transpose(3, 4) - (do * o).sum(4, keepdim=True))
        out.append(packed((ds @ kp) * scale).to(dt))
        for w, x, f in ((ds, qp, scale), (pr, do, 1.0)):
            g = (w.transpose(3, 4) @ x) * f                              # [B, nb, Hk, K, d]
            g = g.permute(0, 1, 3, 2, 4).reshape(-1, Hk, d)
            out.append(torch.zeros_like(k).index_add_(0, rk.reshape(-1), g).to(dt))
    return out


def run(st):
    if not own:
        return plain_qknorm(st) if st["op"] == "qknorm" else plain_window(st)
    from paper_2609_23169_gb300 import ultratex as u
    if st["op"] == "window":
        how = {"left": st["left"], "right": st["right"], "sinks": st["sinks"], "cu_q": st["cu_q"], "cu_k": st["cu_k"],
               "k_len": st["k_len"], "key_mask": st["key_mask"]}
        o, lse = u.ut_window_attn_fwd(st["q"], st["k"], st["v"], **how)
        if not st["train"]:
            return [o, lse]
        return [o, lse, *u.ut_window_attn_bwd(st["q"], st["k"], st["v"], o, lse, st["dout"], **how)]
    d = st["d"]
    rope = u.rope_config(SIDE, axes(d), THETA, TEXT) if st["kind"] == "canvas" else u.rope_config(1, (d, 0, 0), THETA)
    how = {"wq": st["wq"], "wk": st["wk"], "eps": EPS, "pos": st["pos"]}
    if st["cap"]:
        return list(u.ut_qk_norm_rope_fwd(st["q"], st["k"], rope, v=st["v"], rows=st["at"], k_out=st["k_cache"],
                                          v_out=st["v_cache"], **how))
    out = list(u.ut_qk_norm_rope_fwd(st["q"], st["k"], rope, **how))
    if st["train"]:
        out += u.ut_qk_norm_rope_bwd(st["q"], st["k"], rope, st["dqo"], st["dko"], **how)
    return out


def visible(case):
    """(pairs of a row and a key it sees, keys that some row sees), without masks."""
    pairs = keys = 0
    for nq, nk in zip(*key_lengths(case)):
        p = np.arange(nk - nq, nk, dtype=np.int64)
        top = np.minimum(nk, p + case["right"] + 1).clip(0)
        low = np.maximum(0, p - case["left"])
        pairs += int((top - np.minimum(low, top) + np.minimum(np.minimum(case["sinks"], low), top)).sum())
        if nq:
            keys += int(top[-1] - min(low[0], top[-1]) + min(case["sinks"], low[0]))
    return pairs, keys


def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    H, Hk, d = case["heads"], case["kv_heads"], case["d"]
    if case["op"] == "qknorm":
        n = case["rows"]
        one = n * (H + Hk) * d  # values of q and k
        small = 4 * n + 8 * d
        if case["train"]:
            return {"bytes": 5 * one * e + small + 8 * d, "flops": 24 * one}
        rows = 2 * n * Hk * d * e + 4 * n if case["cap"] else 0
        return {"bytes": 2 * one * e + small + rows, "flops": 8 * one}
    pairs, keys = visible(case)
    keep = 0.9 if case["mask"] else 1.0
    qo, kv = case["n_q"] * H * d * e, 2 * keys * Hk * d * e
    small = 4 * case["n_q"] * H + 12 * (case["segs"] + 1) + (keys if case["mask"] else 0)
    if case["train"]:
        return {"bytes": 4 * qo + 2 * kv + small, "flops": 14 * H * d * pairs * keep}
    return {"bytes": 2 * qo + kv + small, "flops": 4 * H * d * pairs * keep}


def exact_qknorm(case, st):
    n, d = case["rows"], case["d"]
    pos = st["pos"].cpu().numpy().astype(np.int64)
    if case["pos"] == "line":
        ang = np.outer(pos.astype(np.float64), [THETA ** (-2.0 * j / d) for j in range(d // 2)])
    else:
        ang = np.zeros((n, d // 2))
        inside = pos >= TEXT
        t = np.where(inside, pos - TEXT, 0)
        at = 0
        for c, a in zip((t // SIDE ** 2, t // SIDE % SIDE, t % SIDE), axes(d)):
            for j in range(a // 2):
                ang[:, at] = c * THETA ** (-2.0 * j / a)
                at += 1
    turn = torch.polar(torch.ones(n, 1, d // 2, dtype=torch.float64, device=st["q"].device),
                       torch.from_numpy(ang).to(st["q"].device)[:, None])

    def of(x, w):
        y = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * w
        y = torch.view_as_complex(y.reshape(n, -1, d // 2, 2)) * turn
        return torch.view_as_real(y).reshape(n, -1, d)

    outs, grads, dws = [], [], []
    for x, w, g in (("q", "wq", "dqo"), ("k", "wk", "dko")):
        x, w = (st[t].double().requires_grad_(case["train"]) for t in (x, w))
        y = of(x, w)
        outs.append(y.detach())
        if case["train"]:
            gx, gw = torch.autograd.grad(y, (x, w), st[g].double())
            grads.append(gx)
            dws.append(gw)
    if case["cap"]:
        kc, vc = st["k_cache"].double(), st["v_cache"].double()
        kc[st["at"].long()], vc[st["at"].long()] = outs[1], st["v"].double()
        return [outs[0], kc, vc]
    return outs + grads + dws


def exact_window(case, st):
    H, Hk, d, n = case["heads"], case["kv_heads"], case["d"], case["n_q"]
    lq, lk = key_lengths(case)
    aq = prefix(lq)
    ak = [s * case["cap"] for s in range(case["segs"])] if case["cap"] else aq
    dev, nk = st["q"].device, st["k"].shape[0]
    z = dict(dtype=torch.float64, device=dev)
    out = [torch.zeros(n, H, d, **z), torch.full((H, n), -math.inf, **z)]
    if case["train"]:
        out += [torch.zeros(n, H, d, **z), torch.zeros(nk, Hk, d, **z), torch.zeros(nk, Hk, d, **z)]
    step = 1024
    for s in range(case["segs"]):
        for r0 in range(0, lq[s], step):
            r1 = min(lq[s], r0 + step)
            i = torch.arange(r0, r1, device=dev)[:, None] + (lk[s] - lq[s])
            low, top = max(0, int(i[0]) - case["left"]), min(lk[s], int(i[-1]) + case["right"] + 1)
            j = torch.arange(lk[s], device=dev)
            j = j[(j < top) & ((j >= low) | (j < case["sinks"]))]
            on = (j <= i + case["right"]) & ((j >= i - case["left"]) | (j < case["sinks"]))
            if st["key_mask"] is not None:
                on = on & (st["key_mask"][ak[s] + j] != 0)
            some = on.any(1)
            if not bool(some.any()):
                continue
            mine = torch.arange(aq[s] + r0, aq[s] + r1, device=dev)[some]
            off = torch.where(on[some], 0.0, -math.inf).double()
            for h in range(H):
                kh = h // (H // Hk)
                q, k, v = st["q"][mine, h].double(), st["k"][ak[s] + j, kh].double(), st["v"][ak[s] + j, kh].double()
                for t in (q, k, v):
                    t.requires_grad_(case["train"])
                sc = q @ k.t() / math.sqrt(d) + off
                o = torch.softmax(sc, 1) @ v
                out[0][mine, h], out[1][h, mine] = o.detach(), torch.logsumexp(sc.detach(), 1)
                if case["train"]:
                    gq, gk, gv = torch.autograd.grad(o, (q, k, v), st["dout"][mine, h].double())
                    out[2][mine, h] = gq
                    out[3][:, kh].index_add_(0, ak[s] + j, gk)
                    out[4][:, kh].index_add_(0, ak[s] + j, gv)
    return out


def exact(case, seed):
    st = prepare(case, seed)
    return exact_qknorm(case, st) if case["op"] == "qknorm" else exact_window(case, st)

"""An attention block over retained tokens with a window: the windowed-attention operators as a model uses them.

    x -> one projection to queries, keys and values -> norms of queries and keys with the position rotation
      -> attention within the window and to the first tokens -> x + (...) Wo

``WindowBlock`` runs it forward and backward over packed segments (training, prompts), and over ``WindowCache``s for new
tokens: their keys and values go straight into the caches.  The projections are plain matrix products.
"""
from __future__ import annotations

from dataclasses import dataclass
from typing import Optional

import torch

from . import ultratex as u


@dataclass
class WindowWeights:
    wqkv: torch.Tensor    # [(H + 2 Hkv) d, C]: queries, keys, values
    norm_q: torch.Tensor  # [d] fp32
    norm_k: torch.Tensor  # [d] fp32
    wo: torch.Tensor      # [C, H d]


class WindowCache:
    """Keys and values of `segments` sequences, `capacity` rows each; their lengths stay on the device.  Calls that are
    given no status word report in the cache's own, which ``ultratex.check_status(cache.status)`` reads."""

    def __init__(self, segments: int, capacity: int, kv_heads: int, head_dim: int, dtype=torch.bfloat16, device="cuda"):
        self.segments, self.capacity = segments, capacity
        self.k = torch.zeros((segments * capacity, kv_heads, head_dim), dtype=dtype, device=device)
        self.v = torch.zeros_like(self.k)
        self.cu = torch.arange(segments + 1, dtype=torch.int32, device=device) * capacity
        self.length = torch.zeros(segments, dtype=torch.int32, device=device)
        self.status = torch.zeros(1, dtype=torch.int32, device=device)

    def place(self, cu_q: torch.Tensor, n: int):
        """Positions [n] and cache rows [n] (int32) of n new tokens in the segments of cu_q.  A segment that has no room
        for all of its new tokens takes none: their rows are behind the caches, which the operators report in the status
        word."""
        return self._place(cu_q, n)[:2]

    def _place(self, cu_q: torch.Tensor, n: int):
        """Positions and rows as place, the lengths [segments] with the new tokens, and which segments have room."""
        length = self.length + (cu_q[1:] - cu_q[:-1])
        room = length <= self.capacity
        token = torch.arange(n, dtype=torch.int32, device=cu_q.device)
        s = torch.bucketize(token, cu_q[1:], right=True, out_int32=True).clamp_(max=self.segments - 1)
        pos = token + (self.length - cu_q[:-1])[s]
        return pos, pos + torch.where(room, self.cu[:-1], self.k.shape[0])[s], length, room


class WindowBlock:
    def __init__(self, heads: int, kv_heads: int, head_dim: int, rope: u.Rope, left: int, right: int = 0, sinks: int = 0,
                 eps: float = 1e-6):
        self.H, self.Hk, self.d, self.rope, self.eps = heads, kv_heads, head_dim, rope, eps
        self.window = {"left": left, "right": right, "sinks": sinks}
        self.saved = None

    def _project(self, x: torch.Tensor, w: WindowWeights):
        qkv = (x @ w.wqkv.t()).view(x.shape[0], self.H + 2 * self.Hk, self.d)
        return qkv[:, :self.H], qkv[:, self.H:self.H + self.Hk], qkv[:, self.H + self.Hk:]

    def forward(self, x: torch.Tensor, w: WindowWeights, pos: Optional[torch.Tensor] = None,
                cu: Optional[torch.Tensor] = None, key_mask: Optional[torch.Tensor] = None,
                status: Optional[torch.Tensor] = None) -> torch.Tensor:
        """x [N, C] with canvas positions pos [N] (default 0, 1, ...), in the segments of cu; key_mask [N]: 0 drops a
        token's key.  Returns [N, C]."""
        q, k, v = self._project(x, w)
        qn, kn = u.ut_qk_norm_rope_fwd(q, k, self.rope, wq=w.norm_q, wk=w.norm_k, eps=self.eps, pos=pos, status=status)
        how = dict(self.window, cu_q=cu, cu_k=cu, key_mask=key_mask, status=status)
        o, lse = u.ut_window_attn_fwd(qn, kn, v, **how)
        self.saved = (x, w, pos, how, q, k, v, qn, kn, o, lse)
        return x + o.flatten(1) @ w.wo.t()

    def backward(self, dy: torch.Tensor):
        """Gradient of the last forward given dy [N, C]: (dx [N, C], gradients of the weights)."""
        x, w, pos, how, q, k, v, qn, kn, o, lse = self.saved
        do = (dy @ w.wo).view(qn.shape)
        dqkv = torch.empty((x.shape[0], self.H + 2 * self.Hk, self.d), dtype=x.dtype, device=x.device)
        dq, dk, dv = dqkv[:, :self.H], dqkv[:, self.H:self.H + self.Hk], dqkv[:, self.H + self.Hk:]
        u.ut_window_attn_bwd(qn, kn, v, o, lse, do, dq=dq, dk=dk, dv=dv, **how)
        _, _, dnq, dnk = u.ut_qk_norm_rope_bwd(q, k, self.rope, dq, dk, wq=w.norm_q, wk=w.norm_k, eps=self.eps, pos=pos,
                                               dq=dq, dk=dk)  # in place
        dqkv = dqkv.flatten(1)
        return dy + dqkv @ w.wqkv, WindowWeights(dqkv.t() @ x, dnq, dnk, dy.t() @ o.flatten(1))

    def extend(self, x: torch.Tensor, w: WindowWeights, cache: WindowCache, cu_q: torch.Tensor,
               pos: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None) -> torch.Tensor:
        """New tokens x [n, C] of the cache's segments (prefix cu_q [segments + 1], on the device), a prompt or single
        tokens: their keys and values are appended, and they attend to what their caches then hold.  pos: canvas
        positions of the rotation, by default those in the sequence.  Of a segment that has no room for all of its new
        tokens none is appended, which is reported in the status word (default: the cache's); they attend to nothing and
        their rows of the result are those of x.  Returns [n, C]."""
        status = cache.status if status is None else status
        q, k, v = self._project(x, w)
        place, rows, length, room = cache._place(cu_q, x.shape[0])
        qn, _, _ = u.ut_qk_norm_rope_fwd(q, k, self.rope, v=v, wq=w.norm_q, wk=w.norm_k, eps=self.eps,
                                         pos=place if pos is None else pos, rows=rows, k_out=cache.k, v_out=cache.v,
                                         status=status)
        torch.where(room, length, cache.length, out=cache.length)
        o, _ = u.ut_window_attn_fwd(qn, cache.k, cache.v, cu_q=cu_q, cu_k=cache.cu, k_len=length * room, status=status,
                                    **self.window)
        return x + o.flatten(1) @ w.wo.t()

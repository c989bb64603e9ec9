"""A conditioning block over the retained tokens of a canvas: the conditioning operators as a model uses them.

    canvas -> retained rows x -> group norm + SiLU per image -> queries
    encoder states -> keys and values (one projection)
    out = x + (cross attention of each image's tokens to its states) Wo -> canvas

``ConditioningBlock`` runs it forward and backward.  The segments are the images: ``image_prefix`` gives the prefix of
their retained tokens on the device, so after the compaction (whose count sizes the problem) nothing returns to the
host.  The projections are plain matrix products.
"""
from __future__ import annotations

from dataclasses import dataclass
from typing import Optional

import torch

from . import ultratex as u


@dataclass
class BlockWeights:
    gamma: torch.Tensor  # [C] fp32
    beta: torch.Tensor   # [C] fp32
    wq: torch.Tensor     # [H d, C]
    wkv: torch.Tensor    # [2 Hkv d, E]: keys, then values
    wo: torch.Tensor     # [C, H d]


def image_prefix(idx: torch.Tensor, images: int, tokens_per_image: int) -> torch.Tensor:
    """Prefix [images + 1] (int32) of the retained tokens of each image, from the ascending canvas positions idx."""
    starts = torch.arange(images + 1, dtype=torch.int32, device=idx.device) * tokens_per_image
    return torch.searchsorted(idx, starts, out_int32=True)


class ConditioningBlock:
    def __init__(self, images: int, tokens_per_image: int, heads: int, kv_heads: int, head_dim: int, groups: int,
                 eps: float = 1e-5):
        self.images, self.tokens_per_image = images, tokens_per_image
        self.H, self.Hk, self.d, self.groups, self.eps = heads, kv_heads, head_dim, groups, eps
        self.saved = None

    def forward(self, mask: torch.Tensor, x: torch.Tensor, states: torch.Tensor, cu_states: torch.Tensor,
                w: BlockWeights, key_mask: Optional[torch.Tensor] = None,
                status: Optional[torch.Tensor] = None) -> torch.Tensor:
        """x [T, C], mask [T] (nonzero = retained), states [M, E] of all images with the prefix cu_states
        [images + 1] and key_mask [M].  Returns the canvas [T, C]; dropped tokens keep their values."""
        idx, n, (xc,) = u.ut_fg_compact(mask, [x], status=status)
        N = int(n.item())
        idx, xc = idx[:N], xc[:N]
        cu = image_prefix(idx, self.images, self.tokens_per_image)
        h, mean, rstd = u.ut_group_norm_fwd(xc, w.gamma, w.beta, self.groups, eps=self.eps, cu=cu, status=status)
        q = (h @ w.wq.t()).view(N, self.H, self.d)
        kv = (states @ w.wkv.t()).view(-1, 2, self.Hk, self.d)
        o, lse = u.ut_xattn_fwd(q, kv[:, 0], kv[:, 1], cu_q=cu, cu_k=cu_states, key_mask=key_mask, status=status)
        y = x.clone()
        u.ut_fg_scatter(idx, N, [xc + o.flatten(1) @ w.wo.t()], [y], u.UT_BG_KEEP)
        self.saved = (mask, idx, xc, cu, h, mean, rstd, q, kv, o, lse, states, cu_states, key_mask, w)
        return y

    def backward(self, dy: torch.Tensor, status: Optional[torch.Tensor] = None):
        """Gradient of the last forward given dy [T, C]: (dx [T, C], dstates [M, E], gradients of the weights)."""
        mask, idx, xc, cu, h, mean, rstd, q, kv, o, lse, states, cu_states, key_mask, w = self.saved
        N = idx.numel()
        dyc = u.ut_fg_compact(mask, [dy], capacity=N, status=status)[2][0]
        do = (dyc @ w.wo).view(q.shape)
        dkv = torch.empty_like(kv)
        dq, _, _ = u.ut_xattn_bwd(q, kv[:, 0], kv[:, 1], o, lse, do, cu_q=cu, cu_k=cu_states, key_mask=key_mask,
                                  dk=dkv[:, 0], dv=dkv[:, 1], status=status)
        dq, dkv = dq.flatten(1), dkv.flatten(1)
        dn, dgamma, dbeta = u.ut_group_norm_bwd(xc, dq @ w.wq, w.gamma, w.beta, mean, rstd, self.groups, cu=cu,
                                                status=status)
        dx = dy.clone()
        u.ut_fg_scatter(idx, N, [dyc + dn], [dx], u.UT_BG_KEEP)
        return dx, dkv @ w.wkv, BlockWeights(dgamma, dbeta, dq.t() @ h, dkv.t() @ states, dyc.t() @ o.flatten(1))

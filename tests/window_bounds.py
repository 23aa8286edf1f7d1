"""Attention whose rows see keys of their own, in 64 bits on the CPU, with the bounds of attn_bounds."""
import math

import torch

from attn_bounds import Ref, U32, _wide


def sees(B, Lq, Lk, window, sinks, start, lens=None, mask=None):
    """B x Lq x Lk truth values; start: a number or one per sequence."""
    start = torch.as_tensor(start).cpu().long().reshape(-1, 1, 1)
    p = start + torch.arange(Lq)[None, :, None]
    j = torch.arange(Lk)[None, None, :]
    ok = (j <= p) & ((j > p - window) | (j < sinks))
    ok = ok.expand(B, Lq, Lk).clone()
    if lens is not None:
        ok &= j < lens.cpu().long().clamp(0, Lk)[:, None, None]
    if mask is not None:
        ok &= (mask.cpu() != 0)[:, None, :]
    return ok


class SeenRef(Ref):
    def __init__(self, Q, K, V, scale, see, tensor=False):
        Lq, dk = Q.shape[1], Q.shape[3]
        Lk, Hkv = K.shape[1], K.shape[2]
        G = Q.shape[2] // Hkv
        self.see, self.ok, self.G, self.scale, self.n, self.dk = see, see.any(dim=1), G, scale, Lk, dk
        self.bf16, self.tensor = Q.dtype == torch.bfloat16, tensor
        used = self.ok[:, None, :, None]
        self.q = _wide(Q, 1)
        self.k, self.v = torch.where(used, _wide(K, G), 0.0), torch.where(used, _wide(V, G), 0.0)
        s = torch.where(see[:, None], self.q @ self.k.transpose(2, 3) * scale, -math.inf)
        if Lk:
            self.lse = torch.logsumexp(s, dim=-1)
        else:
            self.lse = torch.full(s.shape[:3], -math.inf, dtype=torch.float64)
        none = self.lse == -math.inf
        self.p = torch.where(none[..., None], 0.0, torch.exp(s - torch.where(none, 0.0, self.lse)[..., None]))
        self.o = self.p @ self.v
        absdot = self.q.abs() @ self.k.abs().transpose(2, 3) * scale * see[:, None]
        big = torch.where(none, 0.0, self.lse.abs())[..., None]
        self.d = absdot * (dk + 4) * U32 + 8 * U32 * (torch.where(see[:, None], s.abs(), 0.0) + big + 1)
        assert self.p.shape[2] == Lq

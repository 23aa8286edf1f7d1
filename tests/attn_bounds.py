"""Cross attention and its gradient in 64 bits on the CPU, with bounds on what correct kernels may be off.

Half a rounding step, relative: u = 2^-24 (fp32), h = 2^-8 (bf16).  The bounds add up:

* logits: a dot product of dk terms in fp32 is off by at most (dk + 4) u sum |q k|, and the factor
  scale log2(e), the subtraction and 2^x take it to d = scale (dk + 4) u sum |q k| + 8 u (|s| + |lse| + 1), the relative
  error of a weight (twice that with the normalisation's);
* sums of n terms in fp32: at most (n + 16) u times the sum of magnitudes, whatever the order (16: rescalings
  count once a tile, and n >= 64 tiles' worth never occurs here);
* weights (and dS) rounded to bf16 on the tensor cores: independent errors of at most h each, so by
  Hoeffding's inequality their weighted sum passes 7 h sqrt(sum of squares) with probability below
  2 exp(-24.5) = 5e-11 per output; the sums of magnitudes bound it for few terms;
* a bf16 output: h |value|; the gradient reads a bf16 O, whose rounding enters <dO, O> the same way.
"""
import math

import torch

U32, H16 = 2.0 ** -24, 2.0 ** -8


def valid_keys(B, Lk, lens, mask):
    ok = torch.ones(B, Lk, dtype=torch.bool)
    if lens is not None:
        ok &= torch.arange(Lk)[None, :] < lens.cpu().long().clamp(0, Lk)[:, None]
    if mask is not None:
        ok &= mask.cpu() != 0
    return ok


def _wide(x, G):
    """B x L x Hkv x w -> B x Hq x L x w in 64 bits."""
    return x.detach().cpu().double().repeat_interleave(G, dim=2).permute(0, 2, 1, 3)


class Ref:
    def __init__(self, Q, K, V, scale, lens=None, mask=None, tensor=False):
        B, Lq, Hq, dk = Q.shape
        Lk, Hkv = K.shape[1], K.shape[2]
        G = Hq // Hkv
        ok = valid_keys(B, Lk, lens, mask)
        self.ok, self.G, self.scale, self.n, self.dk = ok, G, scale, Lk, dk
        self.bf16, self.tensor = Q.dtype == torch.bfloat16, tensor
        w = ok[:, None, :, None]
        self.q = _wide(Q, 1)
        self.k, self.v = torch.where(w, _wide(K, G), 0.0), torch.where(w, _wide(V, G), 0.0)
        s = self.q @ self.k.transpose(2, 3) * scale
        s = torch.where(ok[:, None, None, :], s, -math.inf)
        self.empty = ~ok.any(dim=1)
        m = s.amax(dim=-1, keepdim=True) if Lk else torch.full((B, Hq, Lq, 1), -math.inf, dtype=torch.float64)
        m = torch.where(m == -math.inf, 0.0, m)
        p = torch.exp(s - m)
        l = p.sum(-1, keepdim=True)
        self.lse = (m + torch.log(l))[..., 0]
        self.p = p / torch.where(l == 0, 1.0, l)
        self.o = self.p @ self.v
        absdot = self.q.abs() @ self.k.abs().transpose(2, 3) * scale
        big = torch.where(torch.isfinite(self.lse), self.lse.abs(), 0.0)[..., None]
        self.d = absdot * (dk + 4) * U32 + 8 * U32 * (torch.where(torch.isfinite(s), s.abs(), 0.0) + big + 1)

    def _rounded(self, w, x):
        """Bound of sum_j round(w_ij) x_j - sum_j w_ij x_j for weights rounded to bf16."""
        if not self.tensor:
            return 0.0
        soft = 7 * H16 * ((w * w) @ (x * x)).sqrt()
        return torch.minimum(soft, H16 * (w.abs() @ x.abs()))

    def _out(self, x, tol):
        return tol + (H16 * (x.abs() + tol) if self.bf16 else U32 * x.abs()) + 1e-37

    def forward_tol(self):
        dmax = self.d.amax(dim=-1, keepdim=True) if self.n else 0.0
        mags = self.p @ self.v.abs()
        tol = (2 * dmax + (2 * self.n + 32) * U32) * mags + self._rounded(self.p, self.v)
        tol_lse = (dmax[..., 0] if self.n else 0.0) + (self.n + 32) * U32 + 4 * U32 * self.lse.abs()
        return self._out(self.o, tol).permute(0, 2, 1, 3), tol_lse

    def grad(self, dO):
        do = _wide(dO, 1)
        dp = do @ self.v.transpose(2, 3)
        D = (do * self.o).sum(-1, keepdim=True)
        ds = self.p * (dp - D)
        n_i, dv = do.shape[2], do.shape[3]
        self.dQ = self.scale * ds @ self.k
        pt, dst = self.p.transpose(2, 3), ds.transpose(2, 3)
        dV, dK = pt @ do, self.scale * dst @ self.q
        # bounds
        od = self.o.abs()
        adp = do.abs() @ self.v.abs().transpose(2, 3)
        e_dp = (dv + 4) * U32 * adp
        e_D = (dv + 4) * U32 * (do.abs() * od).sum(-1, keepdim=True)
        soft = 7 * H16 * ((do * do) * (self.o * self.o)).sum(-1, keepdim=True).sqrt()
        e_round = torch.minimum(soft, H16 * (do.abs() * od).sum(-1, keepdim=True)) if self.bf16 else \
            U32 * (do.abs() * od).sum(-1, keepdim=True)
        e_ds = ds.abs() * (2 * self.d + 8 * U32) + self.p * (e_dp + e_D + 4 * U32 * (dp.abs() + D.abs()))
        t_q = self.scale * (e_ds @ self.k.abs() + (self.n + 32) * U32 * (ds.abs() @ self.k.abs()) +
                            e_round * (self.p @ self.k).abs() * 1.01 + self._rounded(ds, self.k))
        t_v = ((2 * self.d + 8 * U32) * self.p).transpose(2, 3) @ do.abs() + \
            (n_i + 32) * U32 * (pt @ do.abs()) + self._rounded(pt, do)
        t_k = self.scale * (e_ds.transpose(2, 3) @ self.q.abs() + (n_i + 32) * U32 * (dst.abs() @ self.q.abs()) +
                            self._rounded(dst, self.q))
        # the roundings of O differ from row to row: one error per row, weighted by P q
        x = (pt * e_round.transpose(2, 3))
        t_k = t_k + self.scale * torch.minimum(7 * ((x * x) @ (self.q * self.q)).sqrt(), x @ self.q.abs())
        B, _, Lk, _ = dV.shape

        def fold(t, square=False):  # over the query heads of a key head
            t = t.view(B, -1, self.G, Lk, t.shape[-1])
            return t.sum(2).permute(0, 2, 1, 3)

        self.dK, self.dV = fold(dK), fold(dV)
        self.dQ = self.dQ.permute(0, 2, 1, 3)
        return {"dQ": (self.dQ, self._out(self.dQ, t_q.permute(0, 2, 1, 3))),
                "dK": (self.dK, self._out(self.dK, fold(t_k))), "dV": (self.dV, self._out(self.dV, fold(t_v)))}


def close(got, want, tol, what):
    got = got.detach().cpu().double()
    assert torch.isfinite(got).all(), f"{what}: not finite"
    over = (got - want).abs() - tol
    assert (over <= 0).all(), f"{what}: {float(over.max()):.3g} over the bound, at {int(over.argmax())} of {tuple(got.shape)}"

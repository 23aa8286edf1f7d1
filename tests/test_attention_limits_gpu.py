"""Cross attention where its documented limits meet: few keys in a long memory, logits past fp32, logits far from 0, empty axes."""
import math

import pytest
import torch

from attn_bounds import Ref, close

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("path", ["simt", "auto"])
@pytest.mark.parametrize("how, n", [("lens", 1), ("lens", 2), ("lens", 8), ("lens", 64), ("holes", 1), ("holes", 2), ("holes", 5),
                                    ("holes", 16), ("both", 3)])
def test_gradient_over_few_keys_of_a_long_memory(gs, n, how, path):
    """What a sequence's gradient may be off does not grow with the padding around its keys.  With few keys, and weights
    that favour one of them, dP - D cancels, and D from a bf16 O would be off by more than dP - D is rounded.  Bounds as for
    memories that end behind the last key: in the 2-norm, roundings of dS (tensor cores) and of the outputs,
    independent and at most h = 2^-8 each, whose mean square is h^2 / 3 or less (1.2 of room for their spread)."""
    g = torch.Generator().manual_seed(100 * n + len(how))
    B, Lq, Lk, H, w = 6, 50, 1500, 4, 64
    Q, K, V, dO = (torch.randn(B, m, h, w, generator=g).mul(f).bfloat16().cuda()
                   for m, h, f in ((Lq, H, 4.0), (Lk, 2, 1.0), (Lk, 2, 1.0), (Lq, H, 1.0)))
    lens = mask = None
    if how == "lens":
        lens = torch.full((B,), n, dtype=torch.int32).cuda()
    else:
        mask = torch.zeros(B, Lk, dtype=torch.bool)
        for b in range(B):
            mask[b, torch.randperm(Lk - 100, generator=g)[:n]] = True
        if how == "both":  # more of the mask behind the lengths
            mask[:, Lk - 100:] = True
            lens = torch.full((B,), Lk - 100, dtype=torch.int32).cuda()
        mask = mask.cuda()
    r = Ref(Q, K, V, 0.125, lens, mask)
    assert (r.ok.sum(1) == n).all()
    K[~r.ok.cuda()], V[~r.ok.cuda()] = math.nan, math.inf
    O, lse = r.o.permute(0, 2, 1, 3).bfloat16().cuda(), r.lse.float().cuda()
    got = gs.cross_attention_backward(Q, K, V, O, lse, dO, 0.125, key_lens=lens, key_mask=mask, path=path)
    gs.stream_status()
    m = 2 if path == "auto" else 1
    for name, (want, _) in r.grad(dO).items():
        off = (got[name].cpu().double() - want).norm()
        if n == 1 and name != "dV":  # P = 1: dS = 0, whatever fp32 leaves of it
            assert off <= 1e-5 * dO.float().norm().cpu() * 64
            continue
        assert off <= 1.2 * (m / 3) ** 0.5 * 2.0 ** -8 * want.norm(), (name, float(off / want.norm()))


@pytest.mark.parametrize("path", ["simt", "auto"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(3, 1, 700, 2, 64), (3, 1, 5000, 2, 128), (3, 40, 300, 2, 64), (3, 3, 5000, 2, 128),
                                   (3, 200, 400, 2, 64), (39, 200, 400, 4, 64)], ids=lambda s: "x".join(map(str, s)))
def test_logits_past_fp32(gs, shape, dtype, path):
    """Dot products of 4 and -4 under a scale of 2e38: +inf makes a row NaN, -inf weighs nothing, and a row of
    nothing else is empty; rows beside them are as they were."""
    B, Lq, Lk, H, w = shape
    dt = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    g = torch.Generator().manual_seed(Lk + w)
    Q, K = torch.zeros(B, Lq, H, w), torch.zeros(B, Lk, H, w)
    V, dO = torch.randn(B, Lk, H, w, generator=g).to(dt).cuda(), torch.randn(B, Lq, H, w, generator=g).to(dt).cuda()
    sign = (torch.arange(B)[:, None, None] + torch.arange(Lq)[:, None] + torch.arange(H) + 2) % 3 - 1  # -1, 0, 1 by row
    Q[..., 0] = sign
    K[..., 0] = -4.0
    zero = torch.rand(B, Lk, generator=g) < 0.3   # logits of 0 in every row
    zero[0] = False                               # none in the first sequence
    zero[1, :Lk - 60] = False                     # and only at the second one's end
    K[..., 0][zero] = 0.0
    Q, K, zero = Q.to(dt).cuda(), K.to(dt).cuda(), zero.cuda()

    def weights(sign):  # B x H x Lq x Lk
        s = sign.cuda().permute(0, 2, 1)[..., None]
        p = ((s == 0) | zero[:, None, None, :]).double()
        return p / p.sum(-1, keepdim=True).clamp(min=1), p.sum(-1)

    out = gs.cross_attention(Q, K, V, 2e38, want_lse=True, path=path)
    gs.stream_status()
    p, n = weights(sign)
    o, lse = out["O"].double().permute(0, 2, 1, 3), out["lse"].double()
    bad = (sign.cuda() < 0).permute(0, 2, 1)      # 4 * 2e38 among the logits
    assert torch.isnan(o[bad]).all() and torch.isnan(lse[bad]).all()
    want = p @ V.double().permute(0, 2, 1, 3)
    # weights of 1 are exact: sums of Lk terms in fp32 (and their rescalings), the division, a bf16 output
    tol = (Lk + 40) * 2.0 ** -24 * (p @ V.double().abs().permute(0, 2, 1, 3)) + (2.0 ** -8 if dt == torch.bfloat16 else 2.0 ** -24) * want.abs() + 1e-37
    assert ((o - want).abs() <= tol)[~bad].all()
    none = ~bad & (n == 0)
    assert none.any() and (o[none] == 0).all() and (lse[none] == -math.inf).all()
    some = ~bad & (n > 0)
    assert ((lse - n.log()).abs() <= 8 * 2.0 ** -24 * (n.log() + 1))[some].all()
    # the gradient, over rows without a NaN among them
    sign = sign.abs()
    Q[..., 0] = sign.to(dt).cuda()
    out = gs.cross_attention(Q, K, V, 2e38, want_lse=True, path=path)
    got = gs.cross_attention_backward(Q, K, V, out["O"], out["lse"], dO, 2e38, path=path)
    gs.stream_status()
    p, n = weights(sign)
    d = dO.double().permute(0, 2, 1, 3)
    want = (p.transpose(2, 3) @ d).permute(0, 2, 1, 3)
    half = 2.0 ** -8 if dt == torch.bfloat16 else 2.0 ** -24
    # a weight 1 / n: lse to 8 u (log n + 1) and its way through the exponential, rounded to bf16 on the tensor cores
    tol = (half + (Lq + 200) * 2.0 ** -24) * (p.transpose(2, 3) @ d.abs()).permute(0, 2, 1, 3) * 1.01 + half * want.abs() + 1e-37
    assert ((got["dV"].double() - want).abs() <= tol).all()
    assert (got["dQ"].permute(0, 2, 1, 3)[n == 0] == 0).all()


@pytest.mark.parametrize("width", [(64, 64), (47, 64), (64, 47), (33, 7)], ids=str)
def test_forced_tensor_path_without_rows_or_keys(gs, width):
    """An empty axis is no matter of layout: zeros come out whatever the width and alignment."""
    dk, dv = width
    Q, K, V, dO = (torch.randn(2, n, 4, w + 1).bfloat16().cuda()[..., 1:] for n, w in ((9, dk), (70, dk), (70, dv), (9, dv)))
    out = gs.cross_attention(Q, K[:, :0], V[:, :0], 0.2, want_lse=True, path="tensor")
    assert (out["O"] == 0).all() and (out["lse"] == -math.inf).all()
    g = gs.cross_attention_backward(Q, K[:, :0], V[:, :0], out["O"], out["lse"], dO, 0.2, path="tensor")
    assert (g["dQ"] == 0).all() and g["dK"].shape[1] == 0
    g = gs.cross_attention_backward(Q[:, :0], K, V, out["O"][:, :0], out["lse"][:, :, :0].contiguous(), dO[:, :0], 0.2, path="tensor")
    assert (g["dK"] == 0).all() and (g["dV"] == 0).all()
    gs.stream_status()
    f = [t.float() for t in (Q, K[:, :0], V[:, :0])]
    with pytest.raises(gs.GramSpaceError, match="UNSUPPORTED"):  # the type is one
        gs.cross_attention(*f, 0.2, path="tensor")


@pytest.mark.parametrize("Lk", [1, 2, 7, 33, 64, 700])
@pytest.mark.parametrize("far", [0.0, 30.0, 300.0])
def test_fp32_gradient_beside_large_logits(gs, far, Lk):
    """Logits that all lie `far` from 0 leave P off by |lse| 2^-24 or so; dP - D is not to be off by as much of dP."""
    g = torch.Generator().manual_seed(Lk + int(far))
    B, Lq, H, w = 5, 20, 3, 16
    Q, K, V, dO = (torch.randn(B, n, H, m, generator=g) for n, m in ((Lq, w), (Lk, w), (Lk, 4), (Lq, 4)))
    Q[..., 0], K[..., 0] = 1.0, far
    Q[..., 1:] *= 3.0
    Q, K, V, dO = (t.cuda() for t in (Q, K, V, dO))
    lens = torch.tensor([Lk, 1, (Lk + 1) // 2, 0, min(Lk, 3)], dtype=torch.int32).cuda()
    r = Ref(Q, K, V, 1.0, lens)
    O, lse = r.o.permute(0, 2, 1, 3).float().cuda(), r.lse.float().cuda()
    got = gs.cross_attention_backward(Q, K, V, O, lse, dO, 1.0, key_lens=lens)
    gs.stream_status()
    for name, (want, tol) in r.grad(dO).items():
        close(got[name], want, tol, name)

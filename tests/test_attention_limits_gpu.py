"""Cross attention where its documented limits meet: few keys in a long memory."""
import math

import pytest
import torch

from attn_bounds import Ref

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

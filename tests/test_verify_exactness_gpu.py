"""Draws of verify_drafts against running sums in 64 bits, not in the kernel's own units."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def probabilities(N, M, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.softmax(2 * torch.randn(N, M, generator=g, dtype=torch.float64), dim=1).float(), g


def lies_at(w, u, j, slack):
    """Whether the j-th entry's part of the running sums of w (64 bits, relative to their total) holds u, or ends within slack of it."""
    run = np.cumsum(w) / w.sum()
    return w[j] > 0 and (run[j - 1] if j else 0.0) - slack <= u < run[j] + slack


@pytest.mark.parametrize("near", [1e-2, 1e-4, 1e-6])
@pytest.mark.parametrize("M", [1000, 32000, 131072])
def test_draws_of_a_rest_that_is_small(gs, M, near):
    """D lies close to P, so that little is left of P - D.  A weight is off by a unit of 2^-44 at most, and so a running sum's share of the
    total by M 2^-44 / sum(w) (the parts before and behind the point cannot both be off by more than their number of units)."""
    N = 64
    P, g = probabilities(N, M, M)
    D = (P.double() * (1 + near * torch.randn(N, M, generator=g, dtype=torch.float64))).float()
    x = (D.double() / P.double()).argmax(dim=1).int().view(N, 1)
    U = torch.rand(N, 2, generator=g)
    U[:, 0] = 1 - 2.0 ** -24  # the draft, which D has larger, is not kept
    P2 = P[:, None].expand(N, 2, M).contiguous()
    out = gs.verify_drafts(P2.cuda(), D[:, None].cuda(), x.cuda(), U.cuda())
    gs.stream_status()
    assert (out["accepted"] == 0).all() and (out["tokens"][:, 1] == -1).all()
    w = np.maximum(P.numpy().astype(np.float64) - D.numpy().astype(np.float64), 0.0)  # (exact: both are fp32 numbers close by)
    for b in range(N):
        slack = M * 2.0 ** -44 / w[b].sum() + M * 2.0 ** -52  # (the second: the 64-bit sums' own rounding)
        assert slack < 0.1, slack
        assert lies_at(w[b], float(U[b, 1]), int(out["tokens"][b, 0]), slack), b


@pytest.mark.parametrize("M", [1000, 131072])
def test_draws_of_the_target(gs, M):
    N = 64
    P, g = probabilities(N, M, M + 1)
    U = torch.rand(N, 1, generator=g)
    out = gs.verify_drafts(P[:, None].cuda(), None, torch.zeros(N, 0, dtype=torch.int32).cuda(), U.cuda())
    gs.stream_status()
    w = P.numpy().astype(np.float64)
    for b in range(N):
        assert lies_at(w[b], float(U[b, 0]), int(out["tokens"][b, 0]), M * 2.0 ** -45 / w[b].sum() + M * 2.0 ** -52), b


def test_a_rest_below_a_unit_counts_as_nothing(gs):
    """What P has above D is 2^-50: the target's row is drawn from, as where nothing is left.  A rest of two units is drawn from."""
    M = 64
    for more, drawn in ((2.0 ** -50, None), (2.0 ** -43, 7)):
        P = torch.full((1, 2, M), 1.0 / M)
        P[0, 0, 7] = 2.0 ** -27
        D = P[:, :1].clone()
        P[0, 0, 7] += more
        D[0, 0, 3] *= 2
        U = torch.full((16, 2), 0.999)
        U[:, 1] = (torch.arange(16) + 0.5) / 16
        out = gs.verify_drafts(P.expand(16, 2, M).cuda(), D.expand(16, 1, M).cuda(), torch.full((16, 1), 3, dtype=torch.int32).cuda(), U.cuda())
        gs.stream_status()
        assert (out["accepted"] == 0).all()
        w = P[0, 0].double().numpy()
        for b in range(16):
            j = int(out["tokens"][b, 0])
            assert j == drawn if drawn is not None else lies_at(w, float(U[b, 1]), j, M * 2.0 ** -44)

"""sample_scores where differences of scores and temperatures are near or below the smallest normal fp32 number."""
import pytest
import torch

from test_sample_gpu import check

pytestmark = pytest.mark.gpu

HOW = [dict(), dict(k=20), dict(p=0.9), dict(p=0.5, k=40), dict(mp=0.2)]


@pytest.mark.parametrize("M", [50, 300, 2000, 9000])
@pytest.mark.parametrize("spread, T", [(3e-38, 2e-38), (2e-38, 1e-38), (1e-39, 4e-40), (2e-42, 1e-42), (1e-30, 3e-31),
                                       (1e-20, 1e-20), (1e-44, 2e-45), (1e-38, 1.0)], ids=str)
def test_tiny_scores(gs, spread, T, M):
    """Weights are exp((s - m) / T) there as well; numbers that are large beside them weigh 0."""
    g = torch.Generator().manual_seed(M)
    S = (torch.randn(9, M, generator=g).double() * spread).float()
    S[1, ::3] = -3e38
    S[2, ::5] = -float("inf")
    S[3] = -S[3].abs()
    S[4, 1:] = -1e-3
    S[5, ::7] = float("nan")
    U = torch.rand(9, generator=g).cuda()
    for how in HOW:
        check(gs, S.cuda(), U, T=T, **how)
    S[6, 1] = 1e-3                    # one score far above the others
    S[7, 1:3] = float("inf")
    S[8] = spread
    for how in HOW:
        check(gs, S.cuda(), U, T=T, **how)

"""Paged attention over values that are not finite: they reach the rows that see them, in their column, and nothing else."""
import math

import pytest
import torch

from test_paged_gpu import DT, make

pytestmark = pytest.mark.gpu

# short requests are whole units of a CTA, long ones come in pieces that are joined
LENS = {"whole": [40, 300], "joined": [700, 3000]}


def put(cache, table, b, j, where, value):
    page = cache.shape[1]
    cache[(int(table[b, j // page]), j % page) + where] = value


@pytest.mark.parametrize("path", ["auto", "simt"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Lq", [1, 6])
@pytest.mark.parametrize("lens", sorted(LENS))
def test_an_infinite_value_goes_to_the_rows_that_see_it(gs, dtype, path, Lq, lens):
    """In its column and nowhere else, whether all rows of a step see its key or some, and whatever the weights are: of scores, all
    equal (a weight of 1 exactly), or next to the smallest there is."""
    n = LENS[lens]
    for how in ("scores", "equal", "faint"):
        Q, Kc, Vc, table, L = make(2, Lq, 8, 2, 64, 72, 16, n, dtype)
        if how != "scores":
            Q.zero_()
            Q[..., 0] = 8.0  # a logit is the key's first entry
            Kc.zero_()
        for window, sinks, back in ((None, 0, 30), (33, 2, 1), (33, 2, 3), (33, 2, 36), (33, 2, n[1])):
            j = n[1] - back
            K, V = Kc.clone(), Vc.clone()
            if how == "faint":
                put(K, table, 1, j, (slice(None), 0), -85.0)  # a weight of 2^-122.6
            ref = gs.paged_attention(Q, K, V, table, L, window=window, sinks=sinks, want_lse=True, path=path)
            p = n[1] - Lq + torch.arange(Lq)
            see = (j <= p) & ((j > p - (window or 2 ** 40)) | (j < sinks))
            assert see.any() or (back == 36 and Lq == 1)
            hit = torch.zeros(2, Lq, 8, 72, dtype=torch.bool)
            hit[1, :, 4:, 70] = see[:, None]
            for bad in (math.inf, -math.inf, math.nan):
                put(V, table, 1, j, (1, 70), bad)
                out = gs.paged_attention(Q, K, V, table, L, window=window, sinks=sinks, want_lse=True, path=path)
                gs.stream_status()
                O, R = out["O"].cpu(), ref["O"].cpu()
                assert O[hit].isnan().all() if math.isnan(bad) else (O[hit] == bad).all(), (how, window, back, bad)
                assert torch.equal(O[~hit], R[~hit]) and torch.isfinite(R).all() and torch.equal(out["lse"], ref["lse"])


@pytest.mark.parametrize("path", ["auto", "simt"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lens", sorted(LENS))
def test_both_infinities_are_no_number(gs, dtype, path, lens):
    n = LENS[lens]
    for Lq in (1, 6):
        Q, Kc, Vc, table, L = make(2, Lq, 8, 2, 64, 64, 16, n, dtype)
        put(Vc, table, 1, n[1] - 30, (0, 9), math.inf)
        put(Vc, table, 1, n[1] - 200, (0, 9), -math.inf)
        O = gs.paged_attention(Q, Kc, Vc, table, L, path=path)["O"].cpu()
        gs.stream_status()
        assert O[1, :, :4, 9].isnan().all()
        O[1, :, :4, 9] = 0
        assert torch.isfinite(O).all()

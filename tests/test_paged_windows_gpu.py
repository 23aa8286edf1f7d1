"""Paged attention whose rows have different windows: what has left some rows' windows may hold anything for these."""
import math

import pytest
import torch

from test_paged_gpu import DT, make
from test_paged_values_gpu import LENS, put

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("path", ["auto", "simt"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lens", sorted(LENS))
def test_keys_that_have_left_some_rows_windows(gs, dtype, path, lens):
    """Row i of six stands at n - 6 + i and sees the keys from n - 37 + i on (window 32): n - 36 and n - 35 are seen by rows 0 to 2 and not by
    rows 3 to 5, in one step of keys with others that all of them see."""
    n = LENS[lens]
    for bad in (math.nan, math.inf, -math.inf, -torch.finfo(DT[dtype]).max):
        for what in ("keys and values", "values"):
            Q, Kc, Vc, table, L = make(2, 6, 8, 2, 128, 128, 16, n, dtype)
            ref = gs.paged_attention(Q, Kc, Vc, table, L, window=32, sinks=2, want_lse=True, path=path)
            rows = [i for i in range(6) if all(j <= n[0] - 38 + i for j in (n[0] - 36, n[0] - 35))]
            assert rows == [3, 4, 5]
            for b in range(2):
                for j in (n[b] - 36, n[b] - 35):
                    put(Vc, table, b, j, (), bad)
                    if what != "values":
                        put(Kc, table, b, j, (), bad)
            out = gs.paged_attention(Q, Kc, Vc, table, L, window=32, sinks=2, want_lse=True, path=path)
            gs.stream_status()
            assert torch.equal(out["O"][:, rows], ref["O"][:, rows]) and torch.equal(out["lse"][:, :, rows], ref["lse"][:, :, rows])
            if not math.isfinite(bad):
                assert not torch.isfinite(out["O"][:, :3]).any()

"""Window attention where one axis is empty and the other long enough that its work would be cut into parts."""
import math

import pytest
import torch

from test_window_gpu import make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("path", ["auto", "simt"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,Lq,Lk,Hq,Hkv,d", [(2, 0, 300, 2, 1, 64), (2, 300, 0, 2, 1, 64), (1, 0, 3000, 4, 4, 40), (1, 3000, 0, 4, 2, 128),
                                              (2, 0, 5000, 8, 2, 128), (2, 5000, 0, 8, 2, 32)])
def test_one_axis_is_empty(gs, B, Lq, Lk, Hq, Hkv, d, dtype, path):
    for window, sinks in ((1000, 0), (5, 3), (None, 0), (70, 200)):
        Q, K, V, dO = make(B, Lq, Lk, Hq, Hkv, d, d, dtype)
        out = gs.window_attention(Q, K, V, window, sinks, want_lse=True, path=path)
        assert (out["O"] == 0).all() and (out["lse"] == -math.inf).all()
        into = {n: torch.full(t.shape, 7, dtype=t.dtype, device="cuda") for n, t in (("dQ", Q), ("dK", K), ("dV", V))}
        got = gs.window_attention_backward(Q, K, V, out["O"], out["lse"], dO, window, sinks, path=path, out=into)
        gs.stream_status()
        assert all((t == 0).all() for t in got.values())

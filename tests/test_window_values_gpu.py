"""What values that are not finite cost window attention on the tensor cores."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


def milliseconds(f, n=7):
    f()
    t = []
    for _ in range(n):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        f()
        b.record()
        b.synchronize()
        t.append(a.elapsed_time(b))
    return sorted(t)[n // 2]


def test_one_infinite_value_does_not_stall_the_call(gs):
    """Its neighbours' rows are taken again side by side: 2.4 times the call without it, where it was 40 times when a warp took them one
    behind the other.  The bound lies between."""
    g = torch.Generator(device="cuda").manual_seed(1)
    Q, K, V = (torch.randn(4, 4096, h, 128, generator=g, device="cuda").bfloat16() for h in (32, 8, 8))
    clean = milliseconds(lambda: gs.window_attention(Q, K, V, 1024, 4))
    ref = gs.window_attention(Q, K, V, 1024, 4)["O"]
    V[0, 1500, 0, 5] = math.inf
    O = gs.window_attention(Q, K, V, 1024, 4)["O"]
    gs.stream_status()
    hit = torch.zeros(4, 4096, 32, 128, dtype=torch.bool, device="cuda")
    hit[0, 1500:2524, :4, 5] = True
    assert (O[hit] == math.inf).all() and torch.isfinite(O[~hit]).all()
    # two results, each off by its rounding and that of its weights, of values below 6
    assert (O[~hit].float() - ref[~hit].float()).abs().max() <= 2 * 2 * 2.0 ** -8 * 6
    assert milliseconds(lambda: gs.window_attention(Q, K, V, 1024, 4)) <= 10 * clean

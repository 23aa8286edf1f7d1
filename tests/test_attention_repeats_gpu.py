"""Cross attention repeats bit for bit, whatever ran before it."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("G", [3, 5, 7, 100])
@pytest.mark.parametrize("Lq", [2, 260])
@pytest.mark.parametrize("w", [64, 128])
def test_groups_that_do_not_divide_a_tile(gs, w, Lq, G):
    """A tile of rows ends with some that no query fills; what other kernels left in shared memory must not reach the
    rows beside them."""
    g = torch.Generator().manual_seed(G + Lq + w)
    B, Lk, Hkv = (3, 1300, 3) if G < 100 else (2, 700, 2)
    Q, K, V, dO = (torch.randn(B, n, h, w, generator=g).bfloat16().cuda() for n, h in ((Lq, Hkv * G), (Lk, Hkv), (Lk, Hkv), (Lq, Hkv * G)))
    want = gs.cross_attention(Q, K, V, want_lse=True)
    gwant = gs.cross_attention_backward(Q, K, V, want["O"], want["lse"], dO)
    for i in range(6):  # queries of other sizes all over shared memory
        other = torch.randn(4, 700, 16, w, generator=g).mul(3.0 ** i).bfloat16().cuda()
        gs.cross_attention(other, other, other)
        gs.cross_attention_backward(other, other, other, other, torch.zeros(4, 16, 700, device="cuda"), other)
        got = gs.cross_attention(Q, K, V, want_lse=True)
        ggot = gs.cross_attention_backward(Q, K, V, want["O"], want["lse"], dO)
        assert all(torch.equal(got[k], want[k]) for k in want), "forward"
        assert all(torch.equal(ggot[k], gwant[k]) for k in gwant), "gradient"
    gs.stream_status()

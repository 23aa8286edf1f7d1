"""A gradient whose lse is held by nobody but the call."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("path", ["simt", "auto"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_lse_of_an_expression(gs, dtype, path):
    """dQ of one column is as large as lse: from torch's allocator it would get the same memory, were that free."""
    g = torch.Generator().manual_seed(3)
    for w in (1, 2, 64):
        Q, K, V, dO = (torch.randn(2, n, 4, w, generator=g).to(dtype).cuda() for n in (400, 50, 50, 400))
        o = gs.cross_attention(Q, K, V, want_lse=True, path=path)
        want = gs.cross_attention_backward(Q, K, V, o["O"], o["lse"], dO, path=path)
        for _ in range(3):
            got = gs.cross_attention_backward(Q, K, V, o["O"].clone(), o["lse"].clone(), dO.clone(), path=path)
            assert all(torch.equal(got[k], want[k]) for k in want)
    gs.stream_status()

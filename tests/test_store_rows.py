"""Rows of a paged cache at the ends of what page_store takes."""
import ctypes

import pytest
import torch

from test_operator_args import g, heads  # noqa: F401


@pytest.mark.parametrize("H,dk,dv", [(1, 2 ** 31 - 1, 1), (1, 1, 2 ** 31 - 1024), (2 ** 20, 2048, 8), (2 ** 21 - 1, 1024, 1)])
@pytest.mark.parametrize("dtype", [0, 1])
def test_rows_whose_last_steps_pass_32_bits_are_refused(g, H, dk, dv, dtype):  # noqa: F811
    h = heads(g, data=16)
    ref = ctypes.byref
    st = g.load_library().gs_page_store(dtype, 1, 1, H, dk, dv, ref(h), ref(h), 16, 1, 2, 4, ref(h), ref(h), None)
    assert st == g.GS_ERR_SHAPE


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_row_of_2_gib_is_stored(gs, dtype):
    """(Its bytes pass 32 bits.)"""
    w = 2 ** 31 // dtype.itemsize
    K = torch.arange(w, dtype=torch.int32, device="cuda").remainder_(251).to(dtype).view(1, 1, 1, w)
    V = torch.ones(1, 1, 1, 1, dtype=dtype, device="cuda")
    Kc, Vc = (torch.zeros(1, 2, 1, n, dtype=dtype, device="cuda") for n in (w, 1))
    gs.page_store(K, V, torch.ones(1, 1, dtype=torch.int32, device="cuda"), Kc, Vc)
    gs.stream_status()
    assert torch.equal(Kc[0, 1], K[0, 0]) and not Kc[0, 0].any()
    assert Vc[0, :, 0, 0].tolist() == [0, 1]

"""Cross attention beside autograd, which does not record it."""
import warnings

import pytest
import torch


def test_inputs_that_ask_for_a_gradient():
    """A gradient that would be lost is spoken of; a call that wants none is not.  (The calls end at the check for host tensors.)"""
    from paper_2608_01528_gb300 import gramspace as g
    t = [torch.zeros(2, n, 4, 8) for n in (5, 7, 7)]
    for i in range(3):
        a = list(t)
        a[i] = a[i].clone().requires_grad_()
        with pytest.warns(UserWarning, match="cross_attention_backward"), pytest.raises(TypeError, match="CUDA"):
            g.cross_attention(*a)
        with warnings.catch_warnings():
            warnings.simplefilter("error")
            with torch.no_grad(), pytest.raises(TypeError, match="CUDA"):
                g.cross_attention(*a)
            with pytest.raises(TypeError, match="CUDA"):
                g.cross_attention(*(x.detach() for x in a))
            with pytest.raises(TypeError, match="CUDA"):  # the gradient itself
                g.cross_attention_backward(*a, torch.zeros(2, 5, 4, 8), torch.zeros(2, 4, 5), torch.zeros(2, 5, 4, 8))

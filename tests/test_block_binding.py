"""Refusals of the binding that come before any device work: every one is a ClearAttnError."""
import pytest
import torch

from paper_2412_16112_amd import autograd as ag
from paper_2412_16112_amd import clear_attn as ca
from paper_2412_16112_amd import clear_block as cb

BF = torch.bfloat16
X, DH, W, PRE = torch.zeros(4, 64, dtype=BF), torch.zeros(4, 72, dtype=BF), torch.zeros(72, 64, dtype=BF), torch.zeros(2, 4, 72)
ONE = torch.tensor(1.0, dtype=BF)  # no axes


@pytest.mark.parametrize("bad", [
    lambda: cb.gated_ff_backward(DH, X, W[0], W[0], PRE), lambda: cb.gated_ff_backward(DH, X, W[None], W[None], PRE), lambda: cb.gated_ff_backward(DH, X, ONE, ONE, PRE),
    lambda: cb.gated_ff_backward(DH, X, W, W[0], PRE), lambda: cb.gated_ff_backward(DH, X, W, W[:64], PRE), lambda: cb.gated_ff_backward(ONE, X, W, W, PRE), lambda: cb.gated_ff_backward(DH, ONE, W, W, PRE),
    lambda: cb.gated_ff(X, W[0], W[0]), lambda: cb.gated_ff(ONE, W, W), lambda: cb.gated_ff(X, W, W, out=ONE), lambda: ag.gated_ff(ONE, W, W), lambda: ag.gated_ff(X, W[0], W[0]),
    lambda: cb.layer_norm(ONE), lambda: ag.layer_norm(ONE), lambda: cb.layer_norm(X, ONE), lambda: ag.layer_norm(X, ONE), lambda: cb.layer_norm_backward(ONE, ONE, None, None, ONE),
    lambda: cb.rotary(ONE, None, torch.zeros(1), torch.zeros(1)), lambda: ag.rotary(ONE, None, torch.zeros(1), torch.zeros(1)),
    lambda: ag.rotary(torch.zeros(1, 1, 1, 2), ONE, torch.zeros(1), torch.zeros(1)),
])
def test_tensors_of_wrong_axes(bad):
    with pytest.raises(ca.ClearAttnError):
        bad()

"""Which gradients the differentiable gated residual gives: exactly those of the inputs that require one, whichever they are, each what the backward call gives."""
import itertools

import pytest
import torch

from paper_2412_16112_amd import autograd as ag
from paper_2412_16112_amd import clear_block as cb

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("wanted", [w for w in itertools.product((True, False), repeat=6) if any(w)], ids=lambda w: "".join("xygwbp"[i] for i in range(6) if w[i]))
def test_gradients_of_some_inputs(wanted):
    g = torch.Generator(device="cuda").manual_seed(5)
    draw = lambda *shape: torch.randn(*shape, generator=g, device="cuda").to(torch.bfloat16)
    inputs = [draw(2, 50, 384), draw(2, 50, 384), draw(2, 384), draw(384), draw(384), draw(384)]
    dr, dh = draw(2, 50, 384), draw(2, 50, 384)
    how = dict(kind="rms", post="rms")
    _, _, stats = cb.residual_norm(*inputs, save_stats=True, **how)
    want = cb.residual_norm_backward(dr, dh, *inputs, stats, **how)
    leaves = [t.clone().requires_grad_(w) for t, w in zip(inputs, wanted)]
    r, h = ag.residual_norm(*leaves, **how)
    torch.autograd.backward([r, h], [dr, dh])
    for name, leaf, w, b in zip(("x", "y", "gate", "weight", "bias", "post_weight"), leaves, wanted, want):
        assert (leaf.grad is not None) == w, name
        assert not w or torch.equal(leaf.grad, b), name

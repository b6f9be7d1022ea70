"""The differentiable entry points on the device: what they keep, and layouts that they take."""
import pytest
import torch

from paper_2412_16112_amd import autograd as ag

pytestmark = pytest.mark.gpu


def test_validation_with_trainable_weights_takes_the_output_alone():
    M, C, F = 2048, 512, 4096
    x = torch.randn(M, C, device="cuda").bfloat16()
    wg, wu = (torch.randn(F, C, device="cuda").bfloat16().requires_grad_() for _ in range(2))
    ag.gated_ff(x[:8], wg, wu)
    torch.cuda.synchronize()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    with torch.no_grad():
        h = ag.gated_ff(x, wg, wu)
    assert torch.cuda.max_memory_allocated() - before <= 1.5 * h.numel() * 2  # (the products are four times the output)
    kept = ag.gated_ff(x, wg, wu)
    assert torch.equal(kept, h) and kept.requires_grad

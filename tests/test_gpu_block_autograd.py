"""The differentiable entry points on the device: what they keep, and layouts that they take."""
import pytest
import torch

from paper_2412_16112_amd import autograd as ag
from paper_2412_16112_amd import clear_block as cb

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


def test_gradients_of_nothing():
    x = torch.zeros(2, 0, 64, device="cuda", dtype=torch.bfloat16).requires_grad_()
    w = torch.ones(64, device="cuda", dtype=torch.bfloat16)
    ag.layer_norm(x, w, w).sum().backward()
    assert x.grad.shape == x.shape
    q = torch.zeros(1, 2, 0, 64, device="cuda", dtype=torch.bfloat16).requires_grad_()
    sum(t.sum() for t in ag.rotary(q, 2 * q, torch.zeros(0, device="cuda", dtype=torch.int64), cb.rotary_frequencies(64, device="cuda"))).backward()
    assert q.grad.shape == q.shape
    weights = [torch.ones(72, 64, device="cuda", dtype=torch.bfloat16) for _ in range(2)]
    for some in (x, x[0]):
        x.grad = None
        ag.gated_ff(some, *weights).sum().backward()
        assert x.grad.shape == x.shape
    pre = torch.zeros(2, 0, 72, device="cuda")
    for need in ((True, False), (False, True), (True, True)):
        dx, dg, du = cb.gated_ff_backward(x.new_empty(0, 72), x[0], *weights, pre, need=need)
        assert (dx is None) != need[0] and (dg is None or not bool(dg.any())) and (du is None) != need[1]
    stats = torch.zeros(2, 2, 0, device="cuda")
    for need in ((True, False, False), (False, True, False), (True, True, True)):
        got = cb.layer_norm_backward(x, x, w, w, stats, need=need)
        assert [t is not None for t in got] == list(need) and all(t is None or not bool(t.any()) for t in got)

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


def test_gated_ff_on_any_layout_of_its_tokens():
    """The last token of every item, rows at odd places, rows that are one: the tokens' layout is no reason to refuse, and a single row has no stride."""
    N, C, F = 512, 2432, 264
    g = torch.Generator(device="cuda").manual_seed(5)
    draw = lambda *s, k=1.0: (k * torch.randn(*s, generator=g, device="cuda")).bfloat16()
    wg, wu = draw(F, C, k=0.03).requires_grad_(), draw(F, C, k=0.02).requires_grad_()
    long = draw(3, N, C)
    room = draw(7, C + 4)
    for x in (long[:1, -1], long[:, -1], long[:1, -1:], long[:, -1:], room[:, 3:C + 3], room[:, :C], long[0, :1].expand(5, C), draw(4, 3 * C)[:, C:2 * C], draw(1, C + 1)[:, 1:],
              draw(C + 1)[1:], draw(2, 3, C).transpose(0, 1)):
        mine, plain = x.detach().requires_grad_(), x.detach().clone(memory_format=torch.contiguous_format).requires_grad_()
        h, want = ag.gated_ff(mine, wg, wu), ag.gated_ff(plain, wg, wu)
        assert h.shape == x.shape[:-1] + (F,) and torch.equal(h, want)
        dh = torch.empty(h.numel() + 1, dtype=h.dtype, device="cuda")[1:].view(h.shape).copy_(draw(*h.shape))  # (2-byte aligned)
        got = torch.autograd.grad(h, (mine, wg, wu), dh)
        assert all(torch.equal(a, b) for a, b in zip(got, torch.autograd.grad(want, (plain, wg, wu), dh.clone())))
        with torch.no_grad():
            assert torch.equal(ag.gated_ff(x, wg, wu), want)
    for x in (long[:1, -1], long[:1, -1:], long[0, -1]):  # nothing to copy
        assert torch.equal(cb.gated_ff(x, wg, wu), cb.gated_ff(x.clone(), wg, wu))
    out = torch.zeros(1, N, F, dtype=long.dtype, device="cuda")
    cb.gated_ff(long[:1, -1], wg, wu, out=out[:, -1])
    assert torch.equal(out[:, -1], cb.gated_ff(long[:1, -1].clone(), wg, wu)) and not bool(out[:, :-1].any())

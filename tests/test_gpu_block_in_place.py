"""Tensors that a call writes into count as changed: a backward pass that saved one raises instead of working on other values than its forward pass."""
import pytest
import torch

from paper_2412_16112_amd import autograd as ag
from paper_2412_16112_amd import clear_block as cb
from paper_2412_16112_amd.optim import AdamW

pytestmark = pytest.mark.gpu


def draw(*shape, dtype=torch.bfloat16):
    return torch.randn(*shape, device="cuda").to(dtype)


def test_a_backward_pass_behind_an_optimizer_step_raises():
    for bits in (32, 8):
        w = draw(64, 64, dtype=torch.float32).requires_grad_()
        x = draw(8, 64, dtype=torch.float32).requires_grad_()
        opt = AdamW([w], state_bits=bits)
        y = (x @ w).sum()
        opt.step([torch.ones_like(w)])
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.backward()
    m, v = cb.adamw_state(w)
    kept = w.detach().clone()
    before = w._version, kept._version
    cb.adamw_step([w], [torch.ones_like(w)], [m], [v], step=1, lr=0.1, masters=[kept])
    assert w._version > before[0] and kept._version > before[1]
    other, theirs = draw(5, dtype=torch.float32), cb.adamw_state(draw(5))
    opt = AdamW([w, other], masters=True)
    before = w._version, kept._version, opt.masters[0]._version, other._version, opt.masters[1]._version
    cb.adamw_step([w, other], [None, torch.ones_like(other)], [m, theirs[0]], [v, theirs[1]], step=2, lr=0.1, masters=[kept, other.clone()])
    opt.step([None, torch.ones_like(other)])
    assert (w._version, kept._version, opt.masters[0]._version) == before[:3]  # (these were not written)
    assert other._version > before[3] and opt.masters[1]._version > before[4]


def test_outputs_that_the_caller_gave():
    N, d = 12, 64
    freqs, places = cb.rotary_frequencies(d, device="cuda"), torch.arange(N, device="cuda")
    x, w = draw(2, N, d), draw(d)
    wg, wu = draw(72, d), draw(72, d)
    for call in (lambda t: cb.rotary(t, None, places, freqs, out_q=t), lambda t: cb.rotary(draw(1, 2, N, d), t, places, freqs, out_k=t), lambda t: cb.layer_norm(t, w, out=t),
                 lambda t: cb.gated_ff(x, wg, wu, out=t)):
        t = draw(1, 2, N, d) if call.__code__.co_names[1] == "rotary" else draw(2, N, 72) if call.__code__.co_names[1] == "gated_ff" else draw(2, N, d)
        one = torch.ones_like(t).requires_grad_()
        y = (one * t).sum()
        before = t._version
        call(t)
        assert t._version > before
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.backward()
    x = draw(2, N, d).requires_grad_()
    h = ag.layer_norm(x, w)
    with torch.no_grad():
        cb.layer_norm(x, w, out=x)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        h.sum().backward()


def test_inference_tensors_have_no_versions():
    with torch.inference_mode():
        t, w = draw(2, 4, 64), draw(64)
        cb.layer_norm(t, w, out=t)
    cb.layer_norm(t, w, out=t)
    cb.gated_ff(draw(8, 64), draw(64, 64), draw(64, 64), out=t.view(8, 64))
    with torch.inference_mode():
        p, g = draw(100), draw(100)
        m, v = cb.adamw_state(p)
    cb.adamw_step([p], [g], [m], [v], step=1, lr=0.1)
    AdamW([p]).step([g])

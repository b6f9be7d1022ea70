"""The differentiable entry points without a GPU: what they hand to the library (replaced here by plain operations on the CPU) and when."""
import contextlib

import pytest
import torch

from paper_2412_16112_amd import autograd as ag
from paper_2412_16112_amd import clear_block as cb
from tests import block_util as ref


@pytest.fixture
def calls(monkeypatch):
    """Plain stand-ins for the library's calls; the list of what was called."""
    made = []

    def rotary(q, k, positions, freqs, interleaved=True, scale=1.0, inverse=False):
        made.append("rotary")
        return tuple(None if t is None else ref.rotary(t, positions, freqs, interleaved, scale, inverse).to(t.dtype) for t in (q, k))

    def layer_norm(x, weight=None, bias=None, eps=1e-6, weight_offset=0.0, save_stats=False):
        made.append("layer_norm, statistics kept" if save_stats else "layer_norm")
        y = ref.layer_norm(x, weight, bias, eps, weight_offset)
        return (y, torch.zeros((2,) + x.shape[:-1])) if save_stats else y

    def gated_ff(x, w_gate, w_up, activation="silu", save_pre=False):
        made.append("gated_ff, products kept" if save_pre else "gated_ff")
        h = ref.activation(x @ w_gate.T, activation) * (x @ w_up.T)
        return (h, torch.zeros(2, x.shape[0], w_gate.shape[0])) if save_pre else h
    monkeypatch.setattr(cb, "rotary", rotary)
    monkeypatch.setattr(cb, "layer_norm", layer_norm)
    monkeypatch.setattr(cb, "gated_ff", gated_ff)
    monkeypatch.setattr(cb, "layer_norm_backward", lambda dy, x, w, b, stats, weight_offset=0.0, need=None: (dy * 2, None if w is None else w * 2, None if b is None else b * 2))
    monkeypatch.setattr(cb, "gated_ff_backward", lambda dh, x, wg, wu, pre, activation="silu", need=None: (x * 2, wg * 2, wu * 2))
    return made


X = torch.randn(6, 8, generator=torch.Generator().manual_seed(0))
W = torch.randn(16, 8, generator=torch.Generator().manual_seed(1))
PLACES = (torch.arange(6).view(1, 1, 6), torch.ones(1, 4, dtype=torch.float64))
ENTRIES = {  # of one tensor that wants gradients
    "rotary": lambda x: ag.rotary(x.view(1, 1, 6, 8), None, *PLACES)[0],
    "rotary, keys too": lambda x: torch.cat(ag.rotary(x.view(1, 1, 6, 8), 2 * x.view(1, 1, 6, 8), *PLACES), 1),
    "layer_norm": lambda x: ag.layer_norm(x, torch.ones(8), torch.zeros(8)),
    "gated_ff": lambda x: ag.gated_ff(x, W, W),
}


@pytest.mark.parametrize("entry", ENTRIES)
def test_a_gradient_of_a_gradient_is_refused(calls, entry):
    """The backward passes are kernels, which have no derivative here: a penalty on a gradient must raise, not lose its term."""
    x = X.clone().requires_grad_()
    y = ENTRIES[entry](x)
    grad, = torch.autograd.grad(y.square().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        (y.sum() + grad.square().sum()).backward()
    x.grad = None
    ENTRIES[entry](x).square().sum().backward()
    assert x.grad is not None


def test_the_attention_refuses_it_too(monkeypatch):
    class Context:
        forward_strided = staticmethod(lambda Q, K, V, lse=None: Q * V)
        backward_strided = staticmethod(lambda Q, K, V, O, dO, lse: (dO * V, torch.zeros_like(K), dO * Q))
    monkeypatch.setattr(ag, "_context", lambda *a: Context)
    monkeypatch.setattr(torch.cuda, "device", lambda d: contextlib.nullcontext())
    x = torch.randn(1, 1, 4, 64).bfloat16().requires_grad_()
    y = ag.clear_attention(x, x.detach(), x.detach(), 0, 2, 2, 1)
    grad, = torch.autograd.grad(y.float().square().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        grad.sum().backward()


@pytest.mark.parametrize("quiet", [torch.no_grad, torch.inference_mode])
def test_nothing_is_kept_without_gradients(calls, quiet):
    """Trainable weights under no_grad: the two products (8 bytes for each output) and the statistics are for a backward pass that never comes."""
    weights = [W.clone().requires_grad_() for _ in range(2)]
    scale = torch.ones(8).requires_grad_()
    with quiet():
        assert not ag.gated_ff(X, *weights).requires_grad and not ag.layer_norm(X, scale).requires_grad
    assert calls == ["gated_ff", "layer_norm"]
    assert not ag.gated_ff(X, W, W).requires_grad and not ag.layer_norm(X, scale.detach()).requires_grad  # nobody wants gradients
    assert calls[2:] == ["gated_ff", "layer_norm"]
    assert ag.gated_ff(X, *weights).requires_grad and ag.layer_norm(X, scale).requires_grad
    assert calls[4:] == ["gated_ff, products kept", "layer_norm, statistics kept"]


def test_the_attention_without_gradients(monkeypatch):
    """Under no_grad nothing is kept for a backward pass, and fp32 tensors, which have none, are not refused because they want gradients elsewhere."""
    kept = []

    class Context:
        forward = staticmethod(lambda Q, K, V: Q * V)
        forward_lse = staticmethod(lambda Q, K, V: kept.append("lse"))

        @staticmethod
        def forward_strided(Q, K, V, lse=None):
            kept.append("nothing" if lse is None else "lse")
            return Q * V
    monkeypatch.setattr(ag, "_context", lambda *a: Context)
    monkeypatch.setattr(torch.cuda, "device", lambda d: contextlib.nullcontext())
    for dtype in (torch.float32, torch.bfloat16):
        x = torch.randn(1, 1, 4, 64).to(dtype).requires_grad_()
        with torch.no_grad():
            assert not ag.clear_attention(x, x, x, 0, 2, 2, 1).requires_grad
    assert kept == ["nothing"]
    assert ag.clear_attention(x, x, x, 0, 2, 2, 1).requires_grad and kept == ["nothing", "lse"]
    with pytest.raises(ag.ca.ClearAttnError):
        ag.clear_attention(x.detach().float().requires_grad_(), x.float(), x.float(), 0, 2, 2, 1)


def test_weights_of_more_items_than_a_backward_pass_takes(calls):
    """What the backward pass would refuse is refused forward, where gradients are wanted."""
    many, scale = torch.zeros(65536, 1, 8), torch.ones(65536, 8)
    with pytest.raises(ag.ca.ClearAttnError) as e:
        ag.layer_norm(many.clone().requires_grad_(), scale)
    assert e.value.status == ag.ca.CLEAR_ERR_UNSUPPORTED
    with pytest.raises(ag.ca.ClearAttnError):
        ag.layer_norm(many, None, scale.clone().requires_grad_())
    assert calls == []
    ag.layer_norm(many, scale)
    ag.layer_norm(many.clone().requires_grad_(), scale[0])
    ag.layer_norm(many[1:].clone().requires_grad_(), scale[1:])
    assert len(calls) == 3

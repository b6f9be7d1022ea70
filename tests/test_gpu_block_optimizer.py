"""The optimizer class: what it counts, checks and keeps.  The step itself is test_gpu_block_adamw's; here it is the oracle, called with each parameter's own numbers."""
import types

import pytest
import torch

from paper_2412_16112_amd import clear_attn as ca
from paper_2412_16112_amd import clear_block as cb
from paper_2412_16112_amd.optim import AdamW
from tests.test_gpu_block_adamw import HYPER, tensors

pytestmark = pytest.mark.gpu


def moved(opt):
    """Copies of all that a step changes."""
    kept = [*opt.params, *opt.exp_avgs, *opt.exp_avg_sqs, *(opt.masters or ()), *(t for pair in opt.scales or () for t in pair)]
    return [t.detach().clone() for t in kept]


@pytest.mark.parametrize("bits", [32, 8])
def test_a_parameter_counts_its_own_updates(bits):
    """The correction 1 - beta^t is for the t gradients that went into a parameter's moments: with another's t its first step would be up to three times too long."""
    params, grads = tensors(torch.bfloat16, seed=21)
    same = [p.clone() for p in params]
    opt = AdamW(params, state_bits=bits, masters=True, **HYPER)
    states, masters, counts = [cb.adamw_state(p, bits) for p in same], [p.float() for p in same], [0] * len(same)
    for turn in range(6):
        given = [None if (i % 3 == 1 and turn < 4) or (i % 4 == 2 and turn % 2) else g.roll(turn) for i, g in enumerate(grads)]
        opt.step(given)
        for i, g in enumerate(given):
            if g is not None:
                counts[i] += 1
                cb.adamw_step([same[i]], [g], [states[i][0]], [states[i][1]], step=counts[i], masters=[masters[i]], scales=[states[i][2]] if bits == 8 else None, **HYPER)
        assert all(torch.equal(a, b) for a, b in zip(params, same)) and all(torch.equal(a, b) for a, b in zip(opt.masters, masters))
    late = AdamW([torch.zeros(300, device="cuda"), torch.zeros(5, device="cuda")], lr=0.25, weight_decay=0.0, eps=0.0, state_bits=bits)
    for _ in range(10):
        late.step([None, torch.ones(5, device="cuda")])
    late.step([torch.full((300,), 7.0, device="cuda"), None])
    # m / (1 - beta1) = g and sqrt(v / (1 - beta2)) = |g|, to a few roundings of fp32: a first step is lr
    assert bool(((late.params[0] + 0.25).abs() <= 8 * 2.0 ** -24).all())


def test_a_refused_step_changes_nothing():
    params, grads = tensors(torch.float32, seed=3, sizes=[100, 300])
    params.append(torch.randn(50, device="cuda").bfloat16())
    grads.append(torch.randn(50, device="cuda").bfloat16())
    opt = AdamW(params, **HYPER)
    opt.step(grads)
    before = moved(opt)
    bad = [dict(lr=float("nan")), dict(lr=-1.0), dict(beta1=1.0), dict(eps=float("inf")), dict(weight_decay=-1.0), dict(grad_scale=torch.ones(())), dict(grad_scale=torch.ones(2, device="cuda")),
           dict(grad_scale=torch.ones((), device="cuda", dtype=torch.bfloat16)), dict(grads=grads[:2]), dict(grads=[grads[0], grads[1].bfloat16(), grads[2]]), dict(grads=[*grads[:2], grads[2].float()])]
    for change in bad:
        with pytest.raises(ca.ClearAttnError):
            opt.step(**dict(dict(grads=grads), **change))
        assert opt.steps == 1 and all(torch.equal(a, b) for a, b in zip(moved(opt), before)), change
    same = AdamW([p.clone() for p in params], **HYPER)
    with pytest.raises(ca.ClearAttnError):
        same.step(grads, lr=float("nan"))
    assert same.steps == 0
    opt.step(grads)
    assert opt.steps == 2


def test_a_scale_that_is_not_everybodys_is_refused_before_anybody_is_updated(monkeypatch):
    """Parameters on several devices: a scale on one of them is no use to the others.  (The second device is played by a table whose parameters say so.)"""
    params, grads = tensors(torch.float32, seed=3, sizes=[100])
    params.append(torch.randn(50, device="cuda").bfloat16())
    grads.append(torch.randn(50, device="cuda").bfloat16())
    opt = AdamW(params, **HYPER)
    before = moved(opt)
    opt._tables[1][1][0] = types.SimpleNamespace(device=torch.device("cuda", 1), dtype=torch.bfloat16, data_ptr=params[1].data_ptr)
    monkeypatch.setattr(cb, "_set_grads", lambda *a: None)
    opt._tables[0][2][:, 1] = grads[0].data_ptr()
    with pytest.raises(ca.ClearAttnError):
        opt.step(grads, grad_scale=torch.ones((), device="cuda"))
    torch.cuda.synchronize()
    assert opt.steps == 0 and all(torch.equal(a, b) for a, b in zip(moved(opt), before))


@pytest.mark.parametrize("masters", [False, True])
@pytest.mark.parametrize("bits", [32, 8])
def test_a_resumed_optimizer_goes_on_bit_for_bit(bits, masters, tmp_path):
    params, grads = tensors(torch.bfloat16, seed=31)
    opt = AdamW(params, state_bits=bits, masters=masters, **HYPER)
    some = lambda turn: [None if i == 2 and turn < 2 else g.roll(turn) for i, g in enumerate(grads)]
    for turn in range(3):
        opt.step(some(turn))
    torch.save({"opt": opt.state_dict(), "params": params}, tmp_path / "kept")
    loaded = torch.load(tmp_path / "kept", weights_only=True)
    other = [p.cuda() for p in loaded["params"]]
    again = AdamW(other, lr=0.5, state_bits=bits, masters=masters)
    again.load_state_dict(loaded["opt"])
    assert again.hyper == opt.hyper and again.steps == opt.steps == 3
    for turn in range(3, 5):
        opt.step(some(turn))
        again.step(some(turn))
    assert all(torch.equal(a, b) for a, b in zip(moved(opt), moved(again)))


def test_a_state_that_does_not_fit_is_refused_whole():
    params, grads = tensors(torch.float32, seed=33, sizes=[300, 20])
    opt = AdamW(params, state_bits=8, **HYPER)
    opt.step(grads)
    before, good = moved(opt), opt.state_dict()
    for change in (dict(state_bits=32), dict(updates=[1]), dict(updates=[1, -1]), dict(exp_avgs=good["exp_avgs"][:1]), dict(exp_avg_sqs=[t.float() for t in good["exp_avg_sqs"]]),
                   dict(exp_avgs=[good["exp_avgs"][0], torch.zeros(21, dtype=torch.int8)]), dict(scales=None), dict(scales=[good["scales"][0]]), dict(masters=[p.clone() for p in params])):
        with pytest.raises(ca.ClearAttnError):
            opt.load_state_dict(dict(good, **change))
        assert all(torch.equal(a, b) for a, b in zip(moved(opt), before)) and opt.steps == 1, change
    with pytest.raises(ca.ClearAttnError):
        opt.load_state_dict({"exp_avgs": []})


def test_states_are_not_replaced_in_silence():
    """A step works on the tensors that were written down: others in their place would be ignored."""
    opt = AdamW([torch.zeros(10, device="cuda")], masters=True, state_bits=8)
    for name in ("exp_avgs", "exp_avg_sqs", "scales", "masters"):
        with pytest.raises(AttributeError):
            setattr(opt, name, [None])
        with pytest.raises(TypeError):
            getattr(opt, name)[0] = None


def test_a_parameter_given_twice_is_refused():
    """Two descriptors of one tensor would be updated side by side, each reading what the other writes."""
    p, g = torch.ones(300, device="cuda"), torch.ones(300, device="cuda")
    other, empty = torch.ones(10, device="cuda"), torch.ones(0, device="cuda")
    for params in ([p, other, p], [p, p.view(3, 100)], [p, p[:100]], [p[200:], p], [p, p[299:]]):
        with pytest.raises(ca.ClearAttnError) as e:
            AdamW(params)
        assert e.value.status == ca.CLEAR_ERR_INVALID_ARG
    states = [cb.adamw_state(p) for _ in range(2)]
    with pytest.raises(ca.ClearAttnError):
        cb.adamw_step([p, p], [g, g], [s[0] for s in states], [s[1] for s in states], step=1, lr=0.1)
    assert bool((p == 1).all()) and bool((other == 1).all())
    AdamW([p[:150], p[150:], empty, empty.clone(), empty]).step([g[:150], g[150:], empty, None, empty])  # neighbours, and nothing several times
    assert bool((p < 1).all())

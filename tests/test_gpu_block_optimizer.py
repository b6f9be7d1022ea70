"""The optimizer class: what it counts, checks and keeps.  The step itself is test_gpu_block_adamw's; here it is the oracle, called with each parameter's own numbers."""
import pytest
import torch

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

"""What the optimizer says the gradients' norm was, with the library's calls put aside (no GPU needed)."""
import numpy as np
import pytest
import torch

from paper_2412_16112_amd import clear_attn as ca
from paper_2412_16112_amd import clear_block as cb
from paper_2412_16112_amd.optim import AdamW


@pytest.fixture
def opt(monkeypatch):
    """An optimizer of two parameters whose norms are 7, 8, 9, ... and whose launches refuse a rate that is negative."""
    norms = iter(torch.arange(7.0, 100.0))

    def launch(table, first, eight, step, lr, *rest):
        if not lr >= 0:
            raise ca.ClearAttnError(ca.CLEAR_ERR_INVALID_ARG, "lr")
    monkeypatch.setattr(cb, "_table", lambda params, *rest: np.zeros((len(params), 8), dtype=np.int64))
    monkeypatch.setattr(cb, "_set_grads", lambda table, params, grads: [i for i, g in enumerate(grads) if g is not None])
    monkeypatch.setattr(cb, "_launch", launch)
    monkeypatch.setattr(cb, "grad_norm", lambda grads, **how: (next(norms), torch.tensor(1.0)))
    return AdamW([torch.zeros(5), torch.zeros(3)])


GRADS = [torch.ones(5), torch.ones(3)]


def test_a_refused_step_leaves_the_norm(opt):
    opt.step(GRADS, max_norm=1.0)
    assert float(opt.grad_norm) == 7 and opt.steps == 1
    with pytest.raises(ca.ClearAttnError):
        opt.step(GRADS, max_norm=1.0, lr=-1.0)
    assert float(opt.grad_norm) == 7 and opt.steps == 1


def test_no_gradients_have_a_norm_of_0(opt):
    opt.step(GRADS, max_norm=1.0)
    opt.step([None, None], max_norm=1.0)
    assert opt.grad_norm.shape == () and opt.grad_norm.dtype == torch.float32 and float(opt.grad_norm) == 0 and opt.steps == 1
    opt.step([None, GRADS[1]], max_norm=1.0)
    assert float(opt.grad_norm) == 8


def test_a_step_without_a_bound_leaves_it(opt):
    opt.step(GRADS)
    assert opt.grad_norm is None
    opt.step(GRADS, max_norm=1.0)
    opt.step(GRADS)
    assert float(opt.grad_norm) == 7

"""The optimizer with a bound for the gradients' norm: what it says the norm was after steps that were refused or had no gradients."""
import math

import pytest
import torch

from paper_2412_16112_amd import clear_attn as ca
from paper_2412_16112_amd.optim import AdamW

pytestmark = pytest.mark.gpu


def test_the_norm_is_that_of_the_last_step_made():
    params = [torch.randn(300, device="cuda"), torch.randn(7, device="cuda").bfloat16()]
    threes, ones = [torch.full_like(p, 3.0) for p in params], [torch.ones_like(p) for p in params]
    opt = AdamW(params, lr=1e-2)
    opt.step(threes, max_norm=1.0)
    first = opt.grad_norm
    assert abs(float(first) - 3 * math.sqrt(307)) <= 3 * math.sqrt(307) * 2.0 ** -23
    before = [t.clone() for t in (*params, *opt.exp_avgs, *opt.exp_avg_sqs)]
    for bad in (dict(lr=math.nan), dict(lr=-1.0), dict(beta1=1.0), dict(max_norm=-1.0), dict(max_norm=math.nan)):
        with pytest.raises(ca.ClearAttnError):
            opt.step(ones, **dict(dict(max_norm=1.0), **bad))
        assert opt.grad_norm is first and opt.steps == 1, bad
        assert all(torch.equal(a, b) for a, b in zip((*params, *opt.exp_avgs, *opt.exp_avg_sqs), before)), bad
    opt.step([None, None], max_norm=1.0)
    assert opt.grad_norm.is_cuda and opt.grad_norm.shape == () and opt.grad_norm.dtype == torch.float32 and float(opt.grad_norm) == 0
    assert opt.steps == 1 and all(torch.equal(a, b) for a, b in zip((*params, *opt.exp_avgs, *opt.exp_avg_sqs), before))
    opt.step([None, ones[1]], max_norm=1.0)
    assert abs(float(opt.grad_norm) - math.sqrt(7)) <= math.sqrt(7) * 2.0 ** -23

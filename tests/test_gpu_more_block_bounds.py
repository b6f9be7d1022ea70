"""The factor that clips gradients at the ends of its range: norms and bounds that are 0 or infinite."""
import math

import pytest
import torch

from paper_2412_16112_amd import clear_block as cb

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", [2, math.inf])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("u", [None, 0.5])
@pytest.mark.parametrize("value,max_norm,share", [(0.0, 0.0, 1.0), (0.0, 1.0, 1.0), (0.0, math.inf, 1.0), (3.0, math.inf, 1.0), (3.0, 0.0, 0.0), (math.inf, 1.0, 0.0), (math.inf, 0.0, 0.0), (math.inf, math.inf, 1.0)])
def test_factor(kind, dtype, u, value, max_norm, share):
    g = torch.zeros(777, device="cuda", dtype=dtype)
    g[500] = value
    scale = None if u is None else torch.tensor(u, device="cuda")
    one = 1.0 if u is None else u
    norm, factor = cb.grad_norm([g], norm_type=kind, max_norm=max_norm, grad_scale=scale)
    assert float(norm) == one * value and float(factor) == one * share
    want = (g.float() * factor).to(dtype)
    assert torch.equal(cb.clip_grads([g], max_norm, norm_type=kind, grad_scale=scale), norm)
    assert torch.equal(g.isnan(), want.isnan()) and torch.equal(g[~want.isnan()], want[~want.isnan()])

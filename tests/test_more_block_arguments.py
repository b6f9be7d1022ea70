"""Arguments of the gradients' norm, clipping and 4-bit products that Python gives a meaning of their own (no GPU needed): each is refused by name or means what it says."""
import pytest
import torch

from paper_2412_16112_amd import clear_attn as ca
from paper_2412_16112_amd import clear_block as cb


def test_clipping_without_a_bound_is_refused():
    """None is no bound for grad_norm; clip_grads has nothing to do without one, and 0 in its place would make every gradient 0."""
    with pytest.raises(ca.ClearAttnError, match="max_norm"):
        cb.clip_grads([torch.zeros(5)], None)

"""Arguments of the gradients' norm, clipping and 4-bit products that Python gives a meaning of their own (no GPU needed): each is refused by name or means what it says."""
import pytest
import torch

from paper_2412_16112_amd import clear_attn as ca
from paper_2412_16112_amd import clear_block as cb


def test_clipping_without_a_bound_is_refused():
    """None is no bound for grad_norm; clip_grads has nothing to do without one, and 0 in its place would make every gradient 0."""
    with pytest.raises(ca.ClearAttnError, match="max_norm"):
        cb.clip_grads([torch.zeros(5)], None)


W4 = cb.MX4(torch.zeros(5, 32, dtype=torch.uint8), torch.zeros(1, 5, 8, dtype=torch.uint8))


@pytest.mark.parametrize("x,bias", [(torch.zeros(3, 64, requires_grad=True), None), (torch.zeros(3, 64, requires_grad=True) * 2, torch.zeros(5)), (torch.zeros(3, 64), torch.zeros(5, requires_grad=True)),
                                    (W4, torch.zeros(5, requires_grad=True))])
def test_a_product_that_would_cut_a_gradient_off_is_refused(x, bias):
    """The product has no backward pass: tensors before it that are to be trained would be left out without a word.  Without gradients the call goes on to look at where its tensors are."""
    with pytest.raises(ca.ClearAttnError, match="gradient"):
        cb.mx_linear(x, W4, bias)
    for off in (torch.no_grad(), torch.inference_mode()):
        with off, pytest.raises(ca.ClearAttnError, match="device"):
            cb.mx_linear(x, W4, bias)
    with pytest.raises(ca.ClearAttnError, match="device"):
        cb.mx_linear(x if isinstance(x, tuple) else x.detach(), W4, None if bias is None else bias.detach())

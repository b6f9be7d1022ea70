"""Layer norm of more rows than one launch can have."""
import pytest
import torch

from paper_2412_16112_amd import clear_block as cb

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,groups", [(torch.bfloat16, 1), (torch.float32, 3)])
def test_rows_beyond_a_launch(dtype, groups):
    rows, C = (2 ** 26 + 11) // groups, 5
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(groups, rows, C, generator=g, device="cuda", dtype=torch.float32).to(dtype)
    w, b = torch.randn(groups, C, generator=g, device="cuda"), torch.randn(groups, C, generator=g, device="cuda")
    y, stats = cb.layer_norm(x, w, b, save_stats=True)
    assert groups * rows > 2 ** 26 - 3
    each = 2 ** 22
    for first in range(0, rows, each):
        part = slice(first, min(first + each, rows))
        want, s = cb.layer_norm(x[:, part].contiguous(), w, b, save_stats=True)
        assert torch.equal(y[:, part], want) and torch.equal(stats[:, :, part], s), first
    cb.layer_norm(x, w, b, out=x)
    assert torch.equal(x, y)

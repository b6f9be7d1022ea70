"""The gated projection's products in every tile shape, whole and with the contraction in parts, at sizes that end inside tiles and inside stages of the contraction."""
import pytest
import torch

from paper_2412_16112_amd import clear_block as cb
from tests.test_gpu_block_gated import check_backward, check_forward, inputs

pytestmark = pytest.mark.gpu

SIZES = [  # tokens, channels, hidden, with the tiles that the costs choose for them
    (600, 72, 264), (100, 1000, 2056),  # forward in the narrowest tiles, dX and dW in 128 x 128 with several stages in flight, of few and of many stages
    (1001, 136, 1032),  # forward in 128 x 128 with several stages in flight, dX and dW so and in parts
    (1001, 72, 1032), (1001, 4104, 264),  # forward and dX in 128 x 128, two a CU
    (1001, 72, 4104), (2049, 4104, 264),  # forward and dX in 256 x 192
    (600, 72, 8200), (3001, 4104, 264), (600, 1000, 4104),  # forward, dX and dW in 256 x 256; dW in 128 x 128, two a CU, in the first
    (2500, 136, 8200), (4609, 136, 4104), (6001, 264, 2056),  # dW in parts of 256 x 256 and of 128 x 128 two a CU, dX in parts of the latter
    (4609, 136, 8200),  # dX in parts of 256 x 192
    (1500, 2432, 6536), (997, 4096, 11272),  # forward in two launches: full rounds of 256 x 256, the rest in 128 x 128
]


@pytest.mark.parametrize("size", SIZES)
def test_every_tile_shape(size):
    M, C, F = size
    x, wg, wu, dh = inputs(M, C, F, seed=M + F)
    act = ["silu", "gelu_tanh", "gelu_erf"][(M + F // 8) % 3]
    h, pre = cb.gated_ff(x, wg, wu, activation=act, save_pre=True)
    assert torch.equal(h, cb.gated_ff(x, wg, wu, activation=act))
    check_forward(x, wg, wu, act, h, pre)
    got = cb.gated_ff_backward(dh, x, wg, wu, pre, activation=act)
    check_backward(dh, x, wg, wu, act, *got)
    again = cb.gated_ff_backward(dh, x, wg, wu, pre, activation=act)
    assert all(torch.equal(a, b) for a, b in zip(got, again))

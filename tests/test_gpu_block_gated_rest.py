"""The forward product in two launches, the rest in the tiles that the other sizes do not have there."""
import pytest

from tests.test_gpu_block_gated_shapes import test_every_tile_shape as check_size

pytestmark = pytest.mark.gpu

REST = [(4367, 2344, 6016), (4678, 896, 5272)]  # in 256 x 192; in 64 x 128


@pytest.mark.parametrize("size", REST)
def test_the_rest_in_other_tiles(size):
    check_size(size)

"""Which kernels the gated projection takes for the sizes of its numerical tests, pinned (launches recorded instead of made, no GPU): a change of the expected costs that sends these
sizes elsewhere would leave forms untested.  A size that moves needs another in its place."""
import ctypes
import shutil

import pytest

from paper_2412_16112_amd import clear_attn as ca
from tests import fake_launch
from tests.test_gpu_block_gated import SIZES
from tests.test_gpu_block_gated_rest import REST
from tests.test_gpu_block_gated_shapes import SIZES as SHAPES
from tests.test_block_launches import i64, lib, ll, ptr  # noqa: F401  (lib is a fixture)

pytestmark = pytest.mark.skipif(shutil.which("hipcc") is None, reason="hipcc not found")

TILES = {"4, 2, 2, 4": "large", "4, 2, 2, 3": "medium", "2, 2, 4, 3": "medium", "2, 2, 2, 2, 64, 2": "pair", "2, 2, 2, 2, 64, 4": "deep", "1, 4, 2, 1": "narrow"}


def name(launch):
    """The tile's name, with the number of parts that the contraction is in."""
    if launch.kernel.startswith("few_tokens_kernel"):
        return "few" + launch.kernel[18:-1]
    shape = launch.kernel[len("tile_kernel<0, "):-1]
    found = [n for key, n in TILES.items() if shape.startswith(key)]
    assert len(found) == 1, launch
    return found[0] + ("/%d" % launch.grid_y if launch.grid_y > 1 else "")


def forms(lib, M, C, F):  # noqa: F811
    """(forward, dX, dWg and dWu) of a size."""
    assert lib.clear_block_gated_ff(*[ptr(i << 40) for i in range(1, 5)], None, i64(M), C, F, i64(C), i64(C), i64(C), i64(F), 0, None) == ca.CLEAR_OK
    forward = "+".join(name(x) for x in fake_launch.launches(lib))
    assert lib.clear_block_gated_ff_backward(*[ptr(i << 40) for i in range(1, 9)], i64(M), C, F, ll(F, C, C, C, C, C, C), 0, ptr(9 << 40), None) == ca.CLEAR_OK
    made = fake_launch.launches(lib)
    assert made[0].kernel == "gated_gradient_kernel"
    tiles = [x for x in made if x.kernel.startswith("tile_kernel")]
    assert [x.kernel[12] for x in tiles] == ["1", "2"] and len(made) == 3 + sum(x.grid_y > 1 for x in tiles)
    return (forward, *map(name, tiles))


EXPECTED = {
    (1, 8, 8): ("few1", "pair", "pair"), (1, 4096, 1000): ("few1", "deep/4", "pair"), (3, 264, 24): ("few1", "pair", "pair"), (16, 72, 40): ("few1", "pair", "pair"),
    (17, 1000, 88): ("few2", "deep", "pair"), (32, 64, 64): ("few2", "pair", "pair"), (33, 512, 136): ("few4", "deep", "pair"), (64, 2432, 72): ("few4", "deep", "pair"),
    (65, 8, 8): ("narrow", "pair", "pair"), (65, 64, 64): ("narrow", "pair", "pair"), (100, 72, 200): ("narrow", "deep", "pair"), (128, 128, 128): ("narrow", "deep", "pair"),
    (129, 136, 264): ("narrow", "deep", "deep"), (257, 520, 328): ("narrow", "deep", "deep"), (300, 2432, 1000): ("narrow", "deep/4", "pair"), (1000, 328, 2056): ("pair", "deep/6", "deep"),
    (2049, 640, 3208): ("large", "deep/3", "deep"), (5000, 264, 2600): ("large", "deep/2", "deep/2"),
    (600, 72, 264): ("narrow", "deep", "deep"), (100, 1000, 2056): ("narrow", "deep/8", "pair"), (1001, 136, 1032): ("deep", "deep/4", "deep/2"), (1001, 72, 1032): ("pair", "deep/4", "deep/2"),
    (1001, 4104, 264): ("narrow", "pair", "deep"), (1001, 72, 4104): ("medium", "deep/15", "deep"), (2049, 4104, 264): ("narrow", "medium", "deep"), (600, 72, 8200): ("large", "deep/16", "deep"),
    (3001, 4104, 264): ("narrow", "large", "deep"), (600, 1000, 4104): ("pair", "deep/6", "large"), (2500, 136, 8200): ("large", "deep/6", "large/3"), (4609, 136, 4104): ("large", "deep/3", "pair/3"),
    (6001, 264, 2056): ("large", "pair/3", "deep/2"), (4609, 136, 8200): ("large", "medium/10", "large/3"), (1500, 2432, 6536): ("large+deep", "deep", "pair"),
    (997, 4096, 11272): ("large+pair", "large/4", "large"),
    (4367, 2344, 6016): ("large+medium", "medium", "large"), (4678, 896, 5272): ("large+narrow", "large/3", "large"),
}


@pytest.mark.parametrize("size", EXPECTED)
def test_forms_of_the_tested_sizes(lib, size):  # noqa: F811
    assert forms(lib, *size) == EXPECTED[size]


def test_every_form_is_tested():
    tested = set(SIZES) | set(SHAPES) | set(REST)
    assert tested == set(EXPECTED)
    whole = lambda at: {f.split("/")[0] for f in (EXPECTED[s][at] for s in tested) if "/" not in f}
    parts = lambda at: {f.split("/")[0] for f in (EXPECTED[s][at] for s in tested) if "/" in f}
    assert {f for f in (EXPECTED[s][0] for s in tested)} == {"few1", "few2", "few4", "narrow", "deep", "pair", "medium", "large", "large+deep", "large+pair", "large+medium", "large+narrow"}
    assert whole(1) == parts(1) == {"deep", "pair", "medium", "large"}
    assert whole(2) == parts(2) == {"deep", "pair", "large"}


def test_where_few_tokens_end(lib):  # noqa: F811
    """The numbers of tokens up to which the weights are streamed, as the documentation gives them."""
    def last(C, F):
        return max(m for m in range(1, 66) if forms(lib, m, C, F)[0].startswith("few"))
    assert (last(1536, 4096), last(2432, 6528), last(4096, 11264)) == (64, 14, 4)

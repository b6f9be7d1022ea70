"""That the sizes of the test of several turns have them: launches recorded instead of made (no GPU)."""
import shutil

import pytest

from paper_2412_16112_amd import clear_attn as ca
from tests import fake_launch
from tests.test_block_launches import f32, i64, lib, ll, ptr  # noqa: F401  (lib is a fixture)
from tests.test_gpu_block_norm_turns import TURNS

pytestmark = pytest.mark.skipif(shutil.which("hipcc") is None, reason="hipcc not found")


def backward(lib, B, N, C, per_item, dtype):  # noqa: F811
    """(waves a row, chunks, whole rows, teams, turns, ragged) of a call's kernel."""
    rc = lib.clear_block_layer_norm_backward(*[ptr(i << 40) for i in range(1, 8)], i64(B), i64(N), C, ll(*[N * C, C] * 3), per_item, f32(0), dtype, dtype, ptr(8 << 40), None)
    assert rc == ca.CLEAR_OK
    made = [x for x in fake_launch.launches(lib) if x.kernel.startswith("norm_backward_kernel")]
    assert len(made) == 1 and made[0].grid_y == (B if per_item else 1)
    team, chunks, whole = map(int, made[0].kernel[:-1].split(", ")[2:])
    teams, rows = made[0].block // 64 // team, N if per_item else B * N
    return team, chunks, whole, teams, rows / (made[0].grid_x * teams), bool(rows % (made[0].grid_x * teams))


@pytest.mark.parametrize("dtype", [ca.CLEAR_BF16, ca.CLEAR_F32])
def test_every_form_goes_through_several_turns(lib, dtype):  # noqa: F811
    forms, ragged = set(), set()
    for shape in TURNS:
        for per_item in (0, 1):
            team, chunks, whole, _, turns, rest = backward(lib, *shape, per_item, dtype)
            assert turns > 1, shape
            if turns > 2:
                forms.add((team, chunks, whole))
                if rest:
                    ragged.add((team, chunks, whole))
    teams = {(1, 1), (1, 2), (2, 2), (2, 3), (4, 2), (4, 3), (8, 2), (8, 3), (8, 4), (1, 3) if dtype == ca.CLEAR_BF16 else (3, 1)}
    assert forms == ragged == {(*f, whole) for f in teams for whole in (0, 1)}


def forward(lib, C, dtype):  # noqa: F811
    """(waves a row, chunks) of a forward call's kernel."""
    rc = lib.clear_block_layer_norm(ptr(1 << 40), None, None, ptr(2 << 40), None, i64(1), i64(1000), C, ll(0, C, 0, C), 0, f32(1e-6), f32(0), dtype, dtype, None)
    assert rc == ca.CLEAR_OK
    made, = fake_launch.launches(lib)
    return tuple(map(int, made.kernel[:-1].split(", ")[2:4]))


def test_waves_of_a_row_forward(lib):  # noqa: F811
    """One wave with five chunks a lane from 2049 to 2560 channels is the faster form for bf16 alone: in fp32 it is 5 to 13 % slower than two with three."""
    for C, bf16, fp32 in ((1, (1, 1), (1, 1)), (1536, (1, 3), (1, 3)), (1537, (2, 2), (2, 2)), (2048, (2, 2), (2, 2)), (2049, (1, 5), (2, 3)), (2432, (1, 5), (2, 3)), (2560, (1, 5), (2, 3)),
                          (2561, (2, 3), (2, 3)), (4096, (2, 4), (2, 4)), (4097, (4, 3), (4, 3)), (8192, (4, 4), (4, 4)), (8193, (8, 3), (8, 3)), (16384, (8, 4), (8, 4))):
        assert forward(lib, C, ca.CLEAR_BF16) == bf16 and forward(lib, C, ca.CLEAR_F32) == fp32, C

"""What the operators around the attention launch, recorded instead of run (no GPU; pointers are numbers that nothing follows)."""
import ctypes
import shutil

import pytest

from paper_2412_16112_amd import clear_attn as ca
from paper_2412_16112_amd import clear_block as cb
from tests import fake_launch

pytestmark = pytest.mark.skipif(shutil.which("hipcc") is None, reason="hipcc not found")
MOST_THREADS = 2 ** 32 - 1  # of a launch, along an axis of its grid
f32, f64, i64, ptr = ctypes.c_float, ctypes.c_double, ctypes.c_longlong, ctypes.c_void_p


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    return fake_launch.build(str(tmp_path_factory.mktemp("fake_launch")))


def ll(*v):
    return (i64 * len(v))(*v)


@pytest.mark.parametrize("dtype", [ca.CLEAR_BF16, ca.CLEAR_F32])
@pytest.mark.parametrize("channels", [1, 64, 512, 1024, 1111, 1536, 1537, 2048, 2432, 3100, 4096, 4097, 8192, 8193, 16384])
@pytest.mark.parametrize("groups,rows", [(1, 77), (2, 9216), (1, 2 ** 23 - 1), (1, 2 ** 23), (1, 2 ** 24), (4, 2 ** 24 + 3), (1, 2 ** 26), (1, 2 ** 31 - 1), (2 ** 31 - 1, 1), (46340, 46340)])
def test_layer_norm_of_any_number_of_rows(lib, groups, rows, channels, dtype):
    """Every row once, in launches that the device can make."""
    rc = lib.clear_block_layer_norm(ptr(1 << 50), None, None, ptr(1 << 50), None, i64(groups), i64(rows), channels, ll(rows * channels, channels, rows * channels, channels), 0,
                                    f32(1e-6), f32(0), dtype, dtype, None)
    made = fake_launch.launches(lib)
    assert rc == ca.CLEAR_OK and made
    done = 0
    for launch in made:
        assert launch.kernel.startswith("norm_forward_kernel<") and launch.grid_x * launch.block <= MOST_THREADS and launch.grid_y == 1 and launch.first == done
        team = int(launch.kernel.split(",")[2])
        done += launch.grid_x * (launch.block // 64 // team)
    assert done - launch.block // 64 // team < groups * rows <= done
    assert len(made) == -(-groups * rows // (MOST_THREADS // launch.block * (launch.block // 64 // team)))


def gated(lib, tokens, ld_x, ld_h):
    rc = lib.clear_block_gated_ff(ptr(1 << 40), ptr(2 << 40), ptr(3 << 40), ptr(4 << 40), None, i64(tokens), 64, 128, i64(ld_x), i64(64), i64(64), i64(ld_h), 0, None)
    return rc, fake_launch.launches(lib)


def gated_backward(lib, tokens, ld):
    rc = lib.clear_block_gated_ff_backward(ptr(1 << 40), ptr(2 << 40), ptr(3 << 40), ptr(4 << 40), ptr(5 << 40), ptr(6 << 40), ptr(7 << 40), ptr(8 << 40), i64(tokens), 64, 128,
                                           ll(*ld), 0, ptr(9 << 40), None)
    return rc, fake_launch.launches(lib)


@pytest.mark.parametrize("stride", [1 << 20, 512 * 2432, (1 << 40) + 4, 100, 8, 0])
def test_the_row_stride_of_a_single_token_means_nothing(lib, stride):
    """The last token of a sequence is a row whose stride is the sequence's length."""
    plain = gated(lib, 1, 64, 128)
    assert plain[0] == ca.CLEAR_OK and plain[1] and gated(lib, 1, stride, stride) == plain
    plain = gated_backward(lib, 1, (128, 64, 64, 64, 64, 64, 64))
    assert plain[0] == ca.CLEAR_OK and gated_backward(lib, 1, (stride, stride, 64, 64, stride, 64, 64)) == plain
    assert gated(lib, 2, stride, 128)[0] != ca.CLEAR_OK and gated(lib, 2, 64, stride)[0] != ca.CLEAR_OK
    assert gated_backward(lib, 1, (128, 64, stride, 64, 64, 64, 64))[0] != ca.CLEAR_OK  # (a weight has rows)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("dtype", [ca.CLEAR_BF16, ca.CLEAR_F32])
def test_adamw_of_any_number_of_elements(lib, dtype, bits):
    """Every element's workgroup once, in launches that the device can make; what has more elements than that is refused."""
    chunk = 4096  # elements of a workgroup
    for sizes in ([1], [2 ** 35], [2 ** 35, 2 ** 35], [2 ** 34 + 1, 2 ** 35 - 1, 7, 2 ** 35], [0, 5, 0], [2 ** 35 - 4096, 2 ** 34, 2 ** 34], list(range(1, 200)), [2 ** 34] * 70):
        table = (cb.AdamWTensor * len(sizes))(*[cb.AdamWTensor(1 << 40, 1 << 41, None, 1 << 42, 1 << 43, 1 << 44, 1 << 45, n) for n in sizes])
        rc = lib.clear_block_adamw(len(sizes), table, dtype, bits, f64(1e-3), f64(0.9), f64(0.99), f64(1e-8), f64(0), i64(1), None, None)
        made = fake_launch.launches(lib)
        assert rc == ca.CLEAR_OK and all(x.grid_x * x.block <= MOST_THREADS and x.grid_x > 0 for x in made)
        assert sum(x.grid_x for x in made) == sum(-(-n // chunk) for n in sizes)
    table = (cb.AdamWTensor * 1)(cb.AdamWTensor(1 << 40, 1 << 41, None, 1 << 42, 1 << 43, 1 << 44, 1 << 45, 2 ** 35 + 1))
    assert lib.clear_block_adamw(1, table, dtype, bits, f64(1e-3), f64(0.9), f64(0.99), f64(1e-8), f64(0), i64(1), None, None) == ca.CLEAR_ERR_UNSUPPORTED

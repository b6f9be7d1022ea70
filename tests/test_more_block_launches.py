"""What the gated residual, the gradients' norm and the operands in 4 bits launch, recorded instead of run (no GPU; pointers are numbers that nothing follows), and their entry points under the host sanitizers
(AddressSanitizer and UndefinedBehaviorSanitizer over 400 000 draws of arguments)."""
import ctypes
import os
import re
import shutil
import subprocess

import pytest

from paper_2412_16112_amd import clear_attn as ca
from paper_2412_16112_amd import clear_block as cb
from tests import fake_launch

pytestmark = pytest.mark.skipif(shutil.which("hipcc") is None, reason="hipcc not found")
MOST_THREADS = 2 ** 32 - 1  # of a launch, along an axis of its grid
f32, f64, i64, ptr = ctypes.c_float, ctypes.c_double, ctypes.c_longlong, ctypes.c_void_p
MORE = ["block_more_api.cpp", "block_residual.hip", "block_grads.hip", "block_mx.hip"]


def test_entry_points_clean_under_asan_and_ubsan(tmp_path):
    exe = str(tmp_path / "more_block_driver")
    cmd = ["hipcc", "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-Wno-unused-command-line-argument",
           "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=undefined", "-x", "hip",
           os.path.join(fake_launch.CSRC, "block_more_api.cpp"), os.path.join(fake_launch.ROOT, "tests", "host_sanitize", "more_block_driver.cpp"), "-o", exe]
    build = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert build.returncode == 0, build.stdout[-4000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    run = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, env=env, timeout=600)
    assert run.returncode == 0, run.stdout[-4000:]
    assert "clean under the sanitizers" in run.stdout and "runtime error" not in run.stdout and "AddressSanitizer" not in run.stdout


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    with pytest.MonkeyPatch.context() as patch:
        patch.setattr(fake_launch, "SOURCES", fake_launch.SOURCES + [os.path.join(fake_launch.CSRC, s) for s in MORE])
        found = fake_launch.build(str(tmp_path_factory.mktemp("fake_launch")))
    found.fake_launches.restype = ctypes.c_char_p
    for name in cb.EXPORTS:
        if name.endswith("_workspace"):
            getattr(found, name).restype = i64
    return found


def launches(lib):
    """(kernel, whole numbers and truth values among its template arguments, grid x, grid y, threads of a workgroup, LDS) of each launch since the last call."""
    out = []
    for line in lib.fake_launches().decode().splitlines():
        name, x, y, block, lds, _ = line.split("|")
        out.append((re.search(r"\d+((?:residual|grad|mx)_[a-z]+_kernel)", name).group(1), tuple(map(int, re.findall(r"L[ib](\d+)E", name))), int(x), int(y), int(block), int(lds)))
    return out


def ll(*v):
    return (i64 * len(v))(*v)


def at(n):
    return ptr((n + 1) << 56)


@pytest.mark.parametrize("dtype", [ca.CLEAR_BF16, ca.CLEAR_F32])
@pytest.mark.parametrize("channels", [1, 64, 512, 513, 1111, 2432, 2560, 2561, 4096, 5000, 6144, 8192])
@pytest.mark.parametrize("groups,rows", [(1, 77), (2, 9216), (1, 2 ** 24), (4, 2 ** 24 + 3), (1, 2 ** 31 - 1), (2 ** 31 - 1, 1)])
def test_residual_of_any_number_of_rows(lib, groups, rows, channels, dtype):
    s = (rows * channels, channels)
    rc = lib.clear_block_residual_norm(at(0), at(1), None, None, None, None, at(2), at(3), None, i64(groups), i64(rows), channels, ll(*s * 4), 0, 0, 1, 0, f32(1e-6), f32(1), f32(0), f32(0), dtype,
                                       dtype, dtype, None)
    made = launches(lib)
    assert rc == ca.CLEAR_OK and made
    done = 0
    for kernel, (post, team), x, y, block, lds in made:
        assert kernel == "residual_forward_kernel" and post == 0 and x * block <= MOST_THREADS and y == 1 and block % (64 * team) == 0 and team * 512 >= channels
        done += x * (block // 64 // team)
    assert done - block // 64 // team < groups * rows <= done


@pytest.mark.parametrize("groups,rows,gate,per_group", [(1, 1, 0, 0), (1, 5000, 0, 0), (4, 700, 1, 0), (4, 700, 0, 1), (300, 3, 1, 1), (65535, 1, 1, 1), (65535, 3, 0, 0)])
@pytest.mark.parametrize("channels", [8, 512, 2432, 4096, 8192])
def test_residual_backward(lib, groups, rows, gate, per_group, channels):
    s = (rows * channels, channels)
    for stream_dtype in (ca.CLEAR_BF16, ca.CLEAR_F32):
        rc = lib.clear_block_residual_norm_backward(*map(at, range(14)), i64(groups), i64(rows), channels, ll(*s * 6), gate, per_group, 1, 2, f32(1), f32(0), f32(0), ca.CLEAR_BF16, stream_dtype,
                                                    ca.CLEAR_BF16, at(14), None)
        (kernel, (post, team), x, y, block, lds), (join, _, jx, jy, jblock, _) = launches(lib)
        sets = groups if gate or per_group else 1
        assert rc == ca.CLEAR_OK and (kernel, join) == ("residual_backward_kernel", "residual_join_kernel") and post == 1 and y == jy == sets <= 65535 and lds <= 128 * 1024 and block <= 1024
        floats = lib.clear_block_residual_norm_workspace(i64(groups), i64(rows), channels, gate, per_group)
        assert x * sets * 4 * channels <= floats and (x <= 256 or sets > 1) and jx * 64 >= channels


def test_gradients_in_launches_of_many_tensors(lib):
    tensors = (cb.Grad * 400)(*[((i + 1) << 44, 7 if i % 3 else 10 ** 8, i % 2) for i in range(400)])
    assert lib.clear_block_grad_norm(400, tensors, 0, f64(1), None, at(100), at(101), at(102), None) == ca.CLEAR_OK
    made = launches(lib)
    assert [m[0] for m in made] == ["grad_norm_kernel"] * 3 + ["grad_factor_kernel"] and all(m[2] == 1024 for m in made[:2]) and made[3][2] == 1
    assert sum(m[2] for m in made[:3]) * 8 == lib.clear_block_grad_norm_workspace(400, tensors)
    assert lib.clear_block_grad_clip(400, tensors, 0, f64(1), None, at(100), None, at(102), None) == ca.CLEAR_OK
    assert [m[0] for m in launches(lib)] == ["grad_norm_kernel"] * 3 + ["grad_clip_kernel"] * 3
    assert lib.clear_block_grad_clip(0, None, 0, f64(1), None, at(100), None, at(102), None) == ca.CLEAR_OK
    assert [m[0] for m in launches(lib)] == ["grad_factor_kernel"]
    assert lib.clear_block_grad_scale(400, tensors, at(100), None) == ca.CLEAR_OK
    assert [m[0] for m in launches(lib)] == ["grad_scale_kernel"] * 3


@pytest.mark.parametrize("rows", [1, 15, 16, 17, 65535 * 16, 65535 * 16 + 1, 2 ** 31 - 1])
@pytest.mark.parametrize("channels", [32, 256, 2432])
def test_quantisation_of_any_number_of_rows(lib, rows, channels):
    for call in (lambda: lib.clear_block_mx_quantize(at(0), at(1), at(2), i64(rows), channels, i64(channels), i64(-(-channels // 32) * 16), i64(8 * rows), 0, None),
                 lambda: lib.clear_block_mx_dequantize(at(0), at(1), at(2), i64(rows), channels, i64(-(-channels // 32) * 16), i64(8 * rows), i64(channels), 1, None)):
        assert call() == ca.CLEAR_OK
        made = launches(lib)
        assert all(m[2] == -(-channels // 256) and m[3] <= 65535 for m in made) and sum(m[3] for m in made) == -(-rows // 16)


def linear(lib, tokens, channels, outputs, quantized):
    rc = lib.clear_block_mx_linear(at(0), at(1) if quantized else None, at(2), at(3), None, at(4), i64(tokens), channels, outputs,
                                   ll(channels // 2 if quantized else channels, 8 * tokens, channels // 2, 8 * outputs, outputs), 0, 0, 0, at(5), None)
    assert rc == ca.CLEAR_OK
    return launches(lib)


LARGE, PAIR, DEEP, SMALL, FLAT = (4, 2, 2, 4, 2), (2, 2, 2, 2, 2), (2, 2, 2, 2, 4), (1, 2, 2, 1, 4), (1, 4, 2, 1, 3)


@pytest.mark.parametrize("tokens,channels,outputs,want", [
    (1, 4096, 11264, [("mx_few_kernel", (1, 1, 8), 704)]), (4, 4096, 11264, [("mx_few_kernel", (1, 4, 8), 704)]), (5, 4096, 11264, ["quantize", ("mx_few_kernel", (1, 1, 8), 704)]),
    (1, 11264, 4096, [("mx_few_kernel", (1, 1, 16), 256)]), (3, 2304, 4096, [("mx_few_kernel", (1, 4, 16), 256)]), (1, 2048, 2048, [("mx_few_kernel", (1, 1, 8), 128)]),
    (17, 4096, 4096, ["quantize", ("mx_few_kernel", (2, 1, 8), 256)]), (32, 4352, 3840, ["quantize", ("mx_few_kernel", (2, 1, 16), 240)]), (17, 4096, 11264, ["quantize", ("mx_tile_kernel", SMALL, 176)]),
    (77, 4096, 11264, ["quantize", ("mx_tile_kernel", FLAT, 176)]), (333, 2432, 7297, ["quantize", ("mx_tile_kernel", DEEP, 174)]), (64, 9728, 2432, ["quantize", ("mx_tile_kernel", SMALL, 38), "join"]),
    (1000, 1536, 4096, ["quantize", ("mx_tile_kernel", DEEP, 256)]), (800, 4096, 6000, ["quantize", ("mx_tile_kernel", PAIR, 329)]), (16717, 2432, 9728, ["quantize", ("mx_tile_kernel", LARGE, 256)]),
    (2 ** 31 - 1, 32, 1, ["quantize"] * 2049 + [("mx_tile_kernel", FLAT, 512)]),
])
def test_forms_of_the_product(lib, tokens, channels, outputs, want):
    made = linear(lib, tokens, channels, outputs, False)
    assert len(made) == len(want)
    for (kernel, numbers, x, y, block, lds), w in zip(made, want):
        if isinstance(w, str):
            assert kernel == "mx_%s_kernel" % w
        else:
            assert (kernel, numbers, x) == w and lds <= 160 * 1024
    assert [m[:3] for m in linear(lib, tokens, channels, outputs, True)] == [m[:3] for m in made if m[0] != "mx_quantize_kernel"] or tokens <= 4

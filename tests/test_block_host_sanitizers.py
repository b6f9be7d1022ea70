"""The C entry points of the operators around the attention under AddressSanitizer + UndefinedBehaviorSanitizer (CPU only): argument checks over
200 000 draws of sizes, strides, pointers and numbers of every kind, with stand-ins for the launchers (tests/host_sanitize/block_driver.cpp)."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2412_16112_amd", "csrc")
HERE = os.path.join(ROOT, "tests", "host_sanitize")


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="hipcc not found")
def test_block_entry_points_clean_under_asan_and_ubsan(tmp_path):
    exe = str(tmp_path / "block_driver")
    cmd = ["hipcc", "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-Wno-unused-command-line-argument",
           "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=undefined", "-x", "hip",
           os.path.join(CSRC, "block_api.cpp"), os.path.join(HERE, "block_driver.cpp"), "-o", exe]
    build = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert build.returncode == 0, build.stdout[-4000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    run = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, env=env, timeout=600)
    assert run.returncode == 0, run.stdout[-4000:]
    assert "clean under the sanitizers" in run.stdout and "runtime error" not in run.stdout and "AddressSanitizer" not in run.stdout

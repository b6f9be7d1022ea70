"""Where the rotary call's tensors may lie: what it lets through against the elements themselves, over layouts of every kind (CPU only, under the host sanitizers;
tests/host_sanitize/rotary_places_driver.cpp)."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2412_16112_amd", "csrc")
HERE = os.path.join(ROOT, "tests", "host_sanitize")


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="hipcc not found")
def test_no_racing_layout_is_let_through(tmp_path):
    exe = str(tmp_path / "rotary_places_driver")
    cmd = ["hipcc", "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-Wno-unused-command-line-argument",
           "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=undefined", "-x", "hip",
           os.path.join(CSRC, "block_api.cpp"), os.path.join(HERE, "rotary_places_driver.cpp"), "-o", exe]
    build = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert build.returncode == 0, build.stdout[-4000:]
    run = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=600)
    assert run.returncode == 0, run.stdout[-4000:]
    assert "none of these among them" in run.stdout and "runtime error" not in run.stdout and "AddressSanitizer" not in run.stdout

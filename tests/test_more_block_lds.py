"""Where the 4-bit product of few tokens keeps them in LDS, as the device compiler lays it out (compiled, not run: no GPU needed)."""
import os
import shutil
import subprocess

import pytest

from tests import fake_launch

SOURCE = """
#include "%s"
template <int N>
using Group = clear::block::DirectGroup<N>;
template <int N>
constexpr bool fits()
{
    // each of a wave's groups, and each token's row in it, is read 16 bytes at a time; a token's scales two at a time
    return alignof(Group<N>) %% 16 == 0 && sizeof(Group<N>) %% 16 == 0 && sizeof(Group<N>::codes[0]) %% 16 == 0 && offsetof(Group<N>, codes) %% 16 == 0 && offsetof(Group<N>, scales) %% 2 == 0 &&
           sizeof(Group<N>::scales[0]) %% 2 == 0;
}
static_assert(fits<1>(), "one token");
static_assert(fits<clear::block::kDirect>(), "several tokens");
"""


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="hipcc not found")
@pytest.mark.parametrize("side", ["--cuda-device-only", "--cuda-host-only"])
def test_tokens_lie_where_wide_reads_want_them(tmp_path, side):
    path = tmp_path / "layout.hip"
    path.write_text("#include <cstddef>\n" + SOURCE % os.path.join(fake_launch.CSRC, "block_mx.hip"))
    run = subprocess.run(["hipcc", "--offload-arch=gfx950", "-std=c++17", "-Wno-invalid-offsetof", side, "-fsyntax-only", str(path)], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert run.returncode == 0, run.stdout[-4000:]

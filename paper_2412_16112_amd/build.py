"""Builds libclear_attn.so (gfx950) in-tree with hipcc.  Run: python -m paper_2412_16112_amd.build"""
import concurrent.futures
import os
import subprocess
import sys
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libclear_attn.so")
SOURCES = ["clear_attn_api.cpp", "schedule.cpp", "launch_shape.cpp", "kernels_bf16.hip", "kernels_bf16_d64.hip", "kernels_f32.hip", "mfma_peak.hip", "band_merge.hip", "kernels_bf16_bwd.hip", "kernels_bf16_bwd_d64.hip", "prologue.hip", "block_api.cpp", "block_rotary.hip", "block_norm.hip", "block_gated.hip", "block_adamw.hip", "block_more_api.cpp", "block_residual.hip", "block_grads.hip", "block_mx.hip"]
FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",  # no packed-fp32 instructions
    "-Wno-unused-command-line-argument", "-Wno-unknown-attributes",
]


def _run(cmd):
    proc = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    out = "\n".join(l for l in proc.stdout.splitlines() if "is not a recognized feature for this target" not in l)
    if proc.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + out)
    return out


def build(verbose=False, extra_flags=()):
    """Compile every source for gfx950, as many at a time as there are processors but at most 8, and link the shared library; extra_flags go to every command.  Always recompiles."""
    tmp = LIB + ".tmp%d" % os.getpid()
    with tempfile.TemporaryDirectory() as objects, concurrent.futures.ThreadPoolExecutor(min(8, os.cpu_count() or 1)) as pool:
        paths = [os.path.join(objects, s + ".o") for s in SOURCES]
        cmds = [["hipcc", *FLAGS, *extra_flags, "-x", "hip", "-c", os.path.join(CSRC, s), "-o", o] for s, o in zip(SOURCES, paths)]
        link = ["hipcc", "--offload-arch=gfx950", "-shared", "-fPIC", "-Wno-unused-command-line-argument", *extra_flags, *paths, "-o", tmp]
        if verbose:
            print("\n".join(" ".join(c) for c in cmds + [link]), flush=True)
        for out in list(pool.map(_run, cmds)) + [_run(link)]:
            if verbose and out.strip():
                print(out)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True, extra_flags=sys.argv[1:]))

"""The library's entry points with launches recorded instead of made (tests/host_sanitize/fake_launch.cpp): built for the host alone, no GPU."""
import collections
import ctypes
import os
import re
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2412_16112_amd", "csrc")
SOURCES = [os.path.join(CSRC, s) for s in ("block_api.cpp", "block_rotary.hip", "block_norm.hip", "block_gated.hip", "block_adamw.hip")]
SOURCES.append(os.path.join(ROOT, "tests", "host_sanitize", "fake_launch.cpp"))

Launch = collections.namedtuple("Launch", "kernel grid_x grid_y block lds first")


def build(folder):
    objects = [os.path.join(folder, os.path.basename(s) + ".o") for s in SOURCES]
    jobs = [subprocess.Popen(["hipcc", "--offload-arch=gfx950", "-O1", "-std=c++17", "-fPIC", "-x", "hip", "--cuda-host-only", "-fuse-cuid=none", "-Wno-unused-command-line-argument", "-c", s, "-o", o],
                             stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True) for s, o in zip(SOURCES, objects)]
    for s, job in zip(SOURCES, jobs):
        out = job.communicate()[0]
        assert job.returncode == 0, s + ": " + out[-4000:]
    lib = os.path.join(folder, "libfake_launch.so")
    # (its own stand-ins, whatever HIP runtime the process has loaded; each file has an unused id of the same name)
    link = subprocess.run(["g++", "-shared", "-Wl,-Bsymbolic", "-Wl,-z,muldefs", "-o", lib, *objects, "-lpthread"], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert link.returncode == 0, link.stdout[-4000:]
    return ctypes.CDLL(lib)


def launches(lib):
    lib.fake_launches.restype = ctypes.c_char_p
    out = []
    for line in lib.fake_launches().decode().splitlines():
        kernel, *numbers = line.split("|")
        out.append(Launch(plain_name(kernel), *map(int, numbers)))
    return out


def plain_name(mangled):
    """kernel<template arguments>, of the types and numbers that these kernels have."""
    name = mangled[mangled.index("_GLOBAL__N_1") + len("_GLOBAL__N_1"):]
    length = re.match(r"\d+", name).group()
    kernel, rest = name[len(length):len(length) + int(length)], name[len(length) + int(length):]
    arguments = []
    if rest.startswith("I"):
        rest = rest[1:]
        while not rest.startswith("E"):
            piece = re.match(r"DF16b|f|i|x|L[ib](\d+)E", rest)
            arguments.append(piece.group(1) or {"DF16b": "bf16", "f": "f32", "i": "i32", "x": "i64"}[piece.group()])
            rest = rest[piece.end():]
    return "%s<%s>" % (kernel, ", ".join(arguments)) if arguments else kernel

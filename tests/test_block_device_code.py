"""The kernels of the operators around the attention as the compiler left them (no GPU needed): what source and results cannot show."""
import os
import re
import subprocess

import pytest

from tests.test_device_code import LLVM, code_objects, instructions, scalars  # noqa: F401  (code_objects is a fixture)


def buffer_hazards(body):
    """LDS-direct buffer loads of one kernel that follow too closely on a write of M0 (one wait state between them) or on a vector instruction's write of
    their descriptor (five); the number of such loads beside them."""
    bad, loads = [], 0
    for at, load in enumerate(body):
        if not (load.startswith("buffer_load") and load.rstrip().endswith("lds")):
            continue
        loads += 1
        base = scalars(load.split(",")[1].strip())
        assert len(base) == 4, load
        states, i = 0, at - 1
        while i >= 0 and states < 5:
            op, _, rest = body[i].partition(" ")
            operands = [x.strip() for x in rest.split(",")]
            if op.startswith("s_") and operands[0] == "m0" and states < 1:
                bad.append((body[i], load))
            if op.startswith("v_") and any(scalars(x) & base for x in (operands[:2] if re.search("_co_|mad_[ui]64|div_scale", op) else operands[:1])):
                bad.append((body[i], load))
            states += int(operands[0]) + 1 if op == "s_nop" else 1
            i -= 1
    return bad, loads


def test_the_scan_sees_a_hazard():
    assert buffer_hazards(["v_readlane_b32 s5, v1, 2", "s_mov_b32 m0, s9", "s_nop 0", "buffer_load_dwordx4 v7, s[4:7], 0 offen lds"])[0]
    assert buffer_hazards(["s_mov_b32 m0, s9", "buffer_load_dwordx4 v7, s[4:7], 0 offen lds"])[0]
    assert buffer_hazards(["v_readlane_b32 s5, v1, 2", "s_mov_b32 m0, s9", "s_nop 3", "buffer_load_dwordx4 v7, s[4:7], 0 offen lds"]) == ([], 1)


def test_wait_states_of_lds_direct_buffer_loads(code_objects):  # noqa: F811
    """The loads are inline asm, which the compiler's hazard recogniser does not look into: a descriptor that is still being written is a wild address."""
    loads = 0
    for path in code_objects:
        for kernel, body in instructions(path):
            bad, n = buffer_hazards(body)
            loads += n
            assert not bad, "%s: %d of %d loads, the first %s" % (kernel, len(bad), n, bad[0])
    assert loads >= 9 * 16  # nine tile kernels


def test_no_scratch_memory(code_objects):  # noqa: F811
    """Every kernel of these operators keeps what it holds in registers."""
    scratch = {}
    for path in code_objects:
        notes = subprocess.run([os.path.join(LLVM, "llvm-readelf"), "--notes", path], check=True, capture_output=True, text=True).stdout
        for kernel in notes.split("- .agpr_count")[1:]:
            name = re.search(r"\.name: +(_Z\w+)\n", kernel).group(1)
            if "5clear5block" in name:
                scratch[name] = int(re.search(r"\.private_segment_fixed_size: +(\d+)", kernel).group(1))
    assert len(scratch) >= 100
    assert not {k: n for k, n in scratch.items() if n}


@pytest.mark.parametrize("text", ["v_pk_add_f32", "v_pk_mul_f32", "v_pk_fma_f32"])
def test_no_packed_fp32(code_objects, text):  # noqa: F811
    for path in code_objects:
        for kernel, body in instructions(path):
            if "5clear5block" in kernel:
                assert not any(line.startswith(text) for line in body), kernel


def test_no_flat_memory_instructions(code_objects):  # noqa: F811
    """A flat instruction takes its address for one in LDS or in memory by the base, before its own offset is added: a base in front of the first element of an array in LDS is
    an address in memory.  Every pointer of these kernels is known to be one or the other."""
    kernels = 0
    for path in code_objects:
        for kernel, body in instructions(path):
            if "5clear5block" in kernel:
                kernels += 1
                assert not any(line.startswith("flat_") for line in body), kernel
    assert kernels >= 100

"""Loads that are written as instructions are not known to the compiler, which then leaves out the wait states that the hardware wants between
a vector instruction's write of a scalar register and a memory instruction that reads it: five, or the load may use the old value.  This goes
through the library's own device code, as it was built here, and counts them."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2603_19289_amd import build as B

ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")
OBJDUMP = os.path.join(ROCM, "llvm", "bin", "llvm-objdump")
WANTED = 5
REGISTERS = re.compile(r"^s(\d+)$|^s\[(\d+):(\d+)\]$")


def registers(operand):
    """The scalar registers that an operand names."""
    m = REGISTERS.match(operand.strip())
    if not m:
        return set()
    return {int(m[1])} if m[1] else set(range(int(m[2]), int(m[3]) + 1))


def split(line):
    name, _, rest = line.strip().partition(" ")
    return name, [o.strip() for o in rest.split(",")] if rest else []


def states(name, operands):
    return int(operands[0], 0) + 1 if name == "s_nop" else 1


def written_by_vector(name, operands):
    if not name.startswith("v_"):
        return set()
    two = "_co_" in name or name.startswith("v_div_scale")
    return set().union(*(registers(o) for o in operands[:2 if two else 1])) if operands else set()


def too_close(lines):
    """(number of loads to LDS, those with a vector write of their descriptor fewer than five wait states before)."""
    code = [split(x) for x in lines]
    loads, bad = 0, []
    for at, (name, operands) in enumerate(code):
        if not (name.startswith("buffer_load") and operands[-1].split()[-1] == "lds"):
            continue
        loads += 1
        descriptor, passed, back = registers(operands[1].split()[0]), 0, at - 1
        assert len(descriptor) == 4, lines[at]
        while passed < WANTED and back >= 0 and not code[back][0].startswith("<"):
            if written_by_vector(*code[back]) & descriptor:
                bad.append((lines[back], lines[at], passed))
            passed += states(*code[back])
            back -= 1
    return loads, bad


def test_the_count_itself():
    load = "buffer_load_dwordx4 v2, s[4:7], 0 offen lds"
    for between, wrong in ((["s_mov_b32 m0, s9", "s_nop 0"], True), (["s_mov_b32 m0, s9", "s_nop 3"], False), (["s_nop 3"], True), (["s_nop 4"], False),
                           (["v_mov_b32_e32 v1, v2"] * 5, False), (["v_mov_b32_e32 v1, v2"] * 4, True)):
        for writes, here in (("v_readfirstlane_b32 s5, v9", True), ("v_readlane_b32 s7, v9, 3", True), ("v_cmp_gt_u32_e64 s[6:7], s8, v4", True),
                             ("v_add_co_u32_e64 v1, s[4:5], v2, v3", True), ("v_readfirstlane_b32 s8, v9", False), ("s_mov_b32 s5, s9", False),
                             ("v_add_u32_e32 v1, s5, v2", False)):
            loads, bad = too_close([writes, *between, load])
            assert loads == 1 and bool(bad) == (wrong and here), (writes, between)


@pytest.mark.skipif(not os.access(OBJDUMP, os.X_OK), reason="no disassembler here")
def test_descriptors_are_there_before_loads_read_them(tmp_path):
    here = shutil.copy(B.LIB, tmp_path / "library")
    subprocess.run([OBJDUMP, "--offloading", here], check=True, cwd=tmp_path, stdout=subprocess.DEVNULL)
    total = 0
    for image in sorted(tmp_path.glob("library.*gfx950*")):
        text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", image.name], check=True, cwd=tmp_path, capture_output=True, text=True).stdout
        lines = [("<" if x.endswith(">:") else "") + x.split("//")[0].strip() for x in text.splitlines() if x.strip()]
        loads, bad = too_close(lines)
        total += loads
        assert not bad, bad[:5]
    assert total > 100                               # the tiles' loads are among them

"""Copies from HBM straight into LDS, as the built libraries issue them (llvm-objdump of their gfx950 code objects).  They are
inline assembly, inside which the compiler inserts no wait states, and the hardware has no interlock for these two
(the CDNA3 instruction set manual's table of manually inserted wait states, which holds for gfx950):

M0, the copy's LDS address, written by a scalar instruction: one wait state before the copy, or the copy may take the M0 of
the one before it and land in another's place.
A scalar register written by a vector instruction (v_readlane, of a spilled one): five before a copy reads it.  One that a
scalar instruction has written since does not count: that instruction waited for it.
"""

import os
import re
import shutil
import subprocess

import pytest

from paper_2608_00029_amd.build import LIB, NOCLAMP_LIB
from test_residency import _code_objects

OBJDUMP = shutil.which("llvm-objdump", path="/opt/rocm/llvm/bin:" + os.environ.get("PATH", ""))


def scalars(operand):
    m = re.fullmatch(r"s(\d+)|s\[(\d+):(\d+)\]", operand)
    return set() if not m else {int(m[1])} if m[1] else set(range(int(m[2]), int(m[3]) + 1))


def faults(assembly):
    """(copies, [copies too close behind what they read]) of a disassembly."""
    copies, bad, before = 0, [], []
    for line in assembly.splitlines():
        if not line.startswith("\t"):
            before = []
            continue
        op, *rest = line.split("//")[0].split(None, 1)
        args = [a.split()[0] for a in rest[0].split(",")] if rest else []
        if "load_lds" in op or (op.startswith("buffer_load") and re.search(r"\blds\b", line)):
            copies += 1
            wanted, states = set().union(*map(scalars, args)), 0
            m0 = False
            for o, a in reversed(before):
                if states >= 5:
                    break
                written = scalars(a[0]) if a and o.startswith(("s_", "v_")) else set()
                if a and a[0] == "m0" and not m0:
                    m0 = True
                    if states < 1:
                        bad.append(line)
                if written & wanted and o.startswith("v_"):
                    bad.append(line)
                wanted -= written
                states += int(a[0]) + 1 if o == "s_nop" else 1
        before.append((op, args))
    return copies, bad


@pytest.mark.parametrize("path", [LIB, NOCLAMP_LIB], ids=os.path.basename)
def test_copies_wait_for_what_they_read(path, tmp_path):
    if OBJDUMP is None:
        pytest.skip("llvm-objdump not found")
    if not os.path.exists(path):
        pytest.skip("not built")
    with open(path, "rb") as f:
        blob = f.read()
    copies, bad = 0, []
    for i, elf in enumerate(_code_objects(blob)):
        co = tmp_path / f"{i}.elf"
        co.write_bytes(elf)
        text = subprocess.run([OBJDUMP, "-d", "--mcpu=gfx950", str(co)], capture_output=True, text=True, check=True).stdout
        n, b = faults(text)
        copies, bad = copies + n, bad + b
    assert copies > 1000
    assert not bad, (len(bad), bad[:3])


def test_planted_faults_are_seen():
    def of(*lines):
        return faults("0000 <k>:\n" + "".join(f"\t{ln}  // 0000: 00\n" for ln in lines))

    copy = "global_load_lds_dwordx4 v1, s[4:5]"
    assert of("s_mov_b32 m0, s2", copy) == (1, [f"\t{copy}  // 0000: 00"])
    assert len(of("s_add_u32 m0, s2, 0x400", "global_load_lds_dwordx4 v[2:3], off")[1]) == 1
    assert len(of("s_mov_b32 m0, s2", "buffer_load_dwordx4 v1, s[8:11], s3 offen lds")[1]) == 1
    assert of("s_mov_b32 m0, s2", "s_nop 0", copy) == (1, [])
    assert of("s_mov_b32 m0, s2", "v_mov_b32_e32 v9, v8", copy) == (1, [])
    assert len(of("v_readlane_b32 s5, v9, 3", "s_mov_b32 m0, s2", "s_nop 0", copy)[1]) == 1
    assert of("v_readlane_b32 s5, v9, 3", "s_mov_b32 m0, s2", "s_nop 3", copy) == (1, [])
    assert of("v_readlane_b32 s5, v9, 3", "s_add_u32 s5, s5, s6", "s_mov_b32 m0, s2", "s_nop 0", copy) == (1, [])
    assert of("v_readlane_b32 s6, v9, 3", "s_mov_b32 m0, s2", "s_nop 0", copy) == (1, [])

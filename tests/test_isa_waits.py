"""The library's own machine code against a rule of the CDNA3/4 instruction set that the hardware does not enforce: between a vector
instruction that writes a scalar register (v_readfirstlane and the like) and a memory instruction of the vector unit that reads it lie
at least five wait states, or the old value may be read.  The compiler keeps the rule for instructions that it makes itself, not for
the loads written out in inline assembly, whose blocks have to bring the wait states along."""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
WAIT_STATES = 5


def scalars(operand):
    """Numbers of the scalar registers that an operand names: s5, s[8:11], vcc."""
    found = set()
    for a, b in re.findall(r"\bs\[(\d+):(\d+)\]", operand):
        found.update(range(int(a), int(b) + 1))
    found.update(int(a) for a in re.findall(r"\bs(\d+)\b", operand))
    if "vcc" in operand:
        found.update(("vcc",))
    return found


def violations(lines):
    """(function, instruction, wait states) of every vector memory instruction too close to what wrote one of its scalar registers;
    in the order of the code, as it runs where no branch is taken."""
    bad, function, written, now, loads = [], "", {}, 0, 0
    for line in lines:
        head = re.match(r"[0-9a-f]+ <(.+)>:", line)
        if head:
            function, written, now = head.group(1), {}, 0
            continue
        text = line.split("//")[0].strip()
        if not text or ":" in text.split(None, 1)[0]:
            continue
        name, _, rest = text.partition(" ")
        operands = [v.strip() for v in rest.split(",")]
        if name.startswith(("buffer_", "global_", "flat_", "scratch_")):
            loads += " lds" in rest
            near = [now - written[r] - 1 for r in scalars(rest) if r in written]
            if near and min(near) < WAIT_STATES:
                bad.append((function, text, min(near)))
        elif name.startswith("v_"):
            for r in scalars(operands[0]):                       # where a vector instruction writes a scalar register, it comes first
                written[r] = now
        elif name.startswith("s_") and operands and not name.startswith(("s_nop", "s_cmp", "s_waitcnt", "s_barrier", "s_branch", "s_cbranch")):
            for r in scalars(operands[0]):                       # written anew by the scalar unit: no hazard
                written.pop(r, None)
        now += int(operands[0], 0) + 1 if name == "s_nop" else 1
    return bad, loads


def test_the_rule_is_read_right():
    code = ["0000 <f>:", "\tv_readfirstlane_b32 s8, v12", "\ts_mov_b32 m0, s3", "\ts_nop 0", "\tbuffer_load_dwordx4 v1, s[8:11], 0 offen lds"]
    assert violations(code) == ([("f", "buffer_load_dwordx4 v1, s[8:11], 0 offen lds", 2)], 1)
    assert violations([*code[:3], "\ts_nop 2", code[4]])[0][0][2] == 4
    assert violations([*code[:3], "\ts_nop 3", code[4]]) == ([], 1)
    assert violations([code[0], code[1], "\ts_mov_b32 s8, s2", *code[2:]]) == ([], 1)
    assert violations([code[0], "\tv_readfirstlane_b32 s12, v12", *code[2:]]) == ([], 1)
    assert len(violations([code[0], "\tv_cmp_gt_u32_e64 s[2:3], v1, v2", "\tglobal_load_dword v1, v2, s[2:3]"])[0]) == 1


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="needs the disassembler")
def test_scalar_registers_settle_before_vector_memory_reads_them(tmp_path):
    from paper_2210_07454_amd import build
    if not os.path.exists(build.SO):
        build.build()
    so = shutil.copy(build.SO, tmp_path)
    subprocess.run([OBJDUMP, "--offloading", os.path.basename(so)], cwd=tmp_path, check=True, capture_output=True)
    bad, loads = [], 0
    for name in sorted(os.listdir(tmp_path)):
        if not name.endswith("gfx950"):
            continue
        text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", name], cwd=tmp_path, check=True, capture_output=True, text=True).stdout
        found, some = violations(text.splitlines())
        bad += found
        loads += some
    assert loads > 100, "no loads to LDS found: is the disassembly read right?"
    assert not bad, f"{len(bad)} of {loads} loads to LDS or others: {bad[:5]}"

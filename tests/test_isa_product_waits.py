"""The library's own machine code against a rule of the CDNA4 instruction set that the hardware does not enforce: between a matrix instruction and
another instruction that reads or writes a register of its result lie as many wait states as the result takes: 18 after a 32x32x2 product of 32-bit
numbers (16 passes), 12 after a 32x32x16 product of 16-bit ones (8 passes).  The compiler keeps the rule along straight code; it has been seen to
break it where a branch is taken right behind the products, which a result shows only in one column of one kernel.  So every path is followed here.
(A product that adds to the same result takes it from the matrix core and need not wait.)"""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
WAIT_STATES = {"v_mfma_f32_32x32x2_f32": 18, "v_mfma_f32_32x32x16_bf16": 12, "v_mfma_f32_32x32x16_f16": 12}


def registers(operand):
    """The vector and accumulation registers that an operand names: v5, a[0:15]."""
    whole = re.match(r"-?\|?([va])(?:(\d+)|\[(\d+):(\d+)\])\|?$", operand)
    if not whole:
        return frozenset()
    lo, hi = (whole[2], whole[2]) if whole[2] else (whole[3], whole[4])
    return frozenset((whole[1], i) for i in range(int(lo), int(hi) + 1))


def functions(lines):
    """(name, [(address, mnemonic, operands, text)]) of every function."""
    out = []
    for line in lines:
        head = re.match(r"([0-9a-f]+) <(.+)>:", line)
        if head:
            out.append((head[2], []))
            continue
        text, _, comment = line.partition("//")
        text = text.strip()
        at = re.match(r"\s*([0-9A-Fa-f]+):", comment)
        if not text or not at or not out:
            continue
        name, _, rest = text.partition(" ")
        # modifiers stand behind the last operand, without a comma
        operands = [v.split()[0] for v in rest.split(",") if v.split()]
        out[-1][1].append((int(at[1], 16), name, operands, text))
    return out


def violations(lines):
    """(function, product, what touches its result too early, wait states between them), over every path; and how many products there are."""
    bad, products = [], 0
    for function, code in functions(lines):
        place = {at: i for i, (at, *_) in enumerate(code)}
        touched = [frozenset().union(*map(registers, operands)) for _, _, operands, _ in code]
        for i, (_, name, operands, text) in enumerate(code):
            if not name.startswith(("v_mfma", "v_smfma")):
                continue
            products += 1
            result, need = registers(operands[0]), WAIT_STATES[name]
            paths, least = [(i + 1, 0)], {}
            while paths:
                j, waited = paths.pop()
                while j < len(code) and waited < need and least.get(j, need) > waited:
                    least[j] = waited
                    at, other, others, what = code[j]
                    if touched[j] & result:
                        if other.startswith("v_mfma") and not (registers(others[1]) | registers(others[2])) & result:
                            if registers(others[0]) >= result:              # the next one's result, which is followed for itself
                                break
                        else:
                            bad.append((function, text, what, waited))
                            break
                    waited += int(others[0], 0) + 1 if other == "s_nop" else 1
                    if other in ("s_endpgm", "s_setpc_b64"):
                        break
                    if other == "s_branch" or other.startswith("s_cbranch"):
                        jump = int(others[0], 0)
                        target = place[at + 4 + 4 * (jump - 65536 if jump >= 32768 else jump)]
                        if other == "s_branch":
                            j = target
                            continue
                        paths.append((target, waited))
                    j += 1
    return bad, products


def assembled(*lines):
    return ["0000000000000000 <f>:", *(f"\t{line} // {4 * i:012X}: 00000000" for i, line in enumerate(lines))]


def test_the_rule_is_read_right():
    product = "v_mfma_f32_32x32x16_f16 v[0:15], v[16:19], v[20:23], v[0:15]"
    f32 = "v_mfma_f32_32x32x2_f32 a[0:15], v16, v17, a[0:15]"
    few = lambda *lines: [(what, waited) for _, _, what, waited in violations(assembled(*lines))[0]]
    assert few(product, "s_nop 10", "v_add_f32_e32 v30, v3, v31") == [("v_add_f32_e32 v30, v3, v31", 11)]
    assert few(product, "s_nop 11", "v_add_f32_e32 v30, v3, v31") == []
    assert few(product, "v_add_f32_e32 v30, v16, v31", "s_nop 9", "ds_write_b32 v31, v15 offset:4") == [("ds_write_b32 v31, v15 offset:4", 11)]
    assert few(f32, "s_nop 15", "v_accvgpr_read_b32 v1, a15") == [("v_accvgpr_read_b32 v1, a15", 16)]
    assert few(f32, "s_nop 15", "s_nop 1", "v_accvgpr_read_b32 v1, a15") == []
    assert few(f32, "s_nop 15", "v_accvgpr_read_b32 v1, a16") == [] and few(f32, "v_mov_b32_e32 v15, v0") == []
    assert few(product, "v_mov_b32_e32 v2, 0") == [("v_mov_b32_e32 v2, 0", 0)]
    # one that adds to the same result starts anew; one that multiplies with it is early
    assert few(product, "s_nop 7", product, "s_nop 7", "v_mov_b32_e32 v40, v0") == [("v_mov_b32_e32 v40, v0", 8)]
    assert few(product, "v_mfma_f32_32x32x16_f16 v[32:47], v[0:3], v[20:23], v[32:47]")[0][1] == 0
    # a branch: four instructions on, where it is taken, and back
    assert few(product, "s_cbranch_scc1 2", "s_nop 15", "s_endpgm", "v_mov_b32_e32 v40, v0", "s_endpgm") == [("v_mov_b32_e32 v40, v0", 1)]
    assert few("v_mov_b32_e32 v40, v0", product, "s_branch 65533", "v_mov_b32_e32 v41, v1") == [("v_mov_b32_e32 v40, v0", 1)]
    assert few(product, "s_cbranch_scc1 1", "s_nop 12", "s_nop 11", "v_mov_b32_e32 v40, v0") == []


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="needs the disassembler")
def test_products_settle_before_their_results_are_touched(tmp_path):
    from paper_2210_07454_amd import build
    if not os.path.exists(build.SO):
        build.build()
    so = shutil.copy(build.SO, tmp_path)
    subprocess.run([OBJDUMP, "--offloading", os.path.basename(so)], cwd=tmp_path, check=True, capture_output=True)
    bad, products = [], 0
    for name in sorted(os.listdir(tmp_path)):
        if not name.endswith("gfx950"):
            continue
        text = subprocess.run([OBJDUMP, "-d", name], cwd=tmp_path, check=True, capture_output=True, text=True).stdout
        if "mfma" in text:
            found, some = violations(text.splitlines())
            bad += found
            products += some
    assert products > 5000, "no matrix instructions found: is the disassembly read right?"
    assert not bad, f"{len(bad)} places: {bad[:5]}"

"""The library's own code for the scan with matrix states, disassembled: where values are split into pairs of fp16, and where lanes are swapped, no vector
instruction takes a matrix instruction's result, or writes over a result or over what is being added to, before the processor is done with it.  The
compiler leaves the wait states between its own instructions; those inside of assembler statements it does not look at.  Host only."""
import os
import re
import shutil
import subprocess

import pytest

import paper_1907_06154_amd as ssam

OBJDUMP = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin", "llvm-objdump")
# wait states behind a matrix instruction's issue: until its result may be read or written over, and until the registers of what it adds to may be
WAITS = {"v_mfma_f32_16x16x32_f16": (8, 3), "v_mfma_f32_16x16x4_f32": (10, 7)}
MOST = max(max(w) for w in WAITS.values())


def registers(operand):
    m = re.match(r"-?\|?([va])(?:\[(\d+):(\d+)\]|(\d+)\b)", operand.strip())
    if not m:
        return set()
    first, last = (m[2], m[3]) if m[2] else (m[4], m[4])
    return {(m[1], i) for i in range(int(first), int(last) + 1)}


def too_early(lines):
    """(vector instruction, matrix instruction, wait states between them) wherever they are too few, on any way through the code."""
    code, labels = [], {}
    for line in lines:
        m = re.match(r"^[0-9a-f]+ <(L\d+)>:", line)
        if m:
            labels[m[1]] = len(code)
        elif line.startswith("\t"):
            name, _, rest = line.split("//")[0].strip().partition(" ")
            code.append((name, rest.split(",")))
    before = [[] for _ in range(len(code) + 1)]
    for i, (name, ops) in enumerate(code):
        if name.startswith(("s_cbranch", "s_branch")):
            before[labels[ops[0].strip()]].append(i)
        if name not in ("s_branch", "s_endpgm"):
            before[i + 1].append(i)
    found = []
    for i, (name, ops) in enumerate(code):
        if not name.startswith(("v_fma_mixlo", "v_fma_mixhi", "v_permlane16_swap", "v_permlane32_swap")):
            continue
        written = registers(ops[0])
        read = written.union(*map(registers, ops[1:]))      # (half of the register stays)
        if "swap" in name:
            written |= registers(ops[1])
        ways, seen = [(j, 0) for j in before[i]], {}
        while ways:
            j, waits = ways.pop()
            if waits >= MOST or seen.get(j, MOST) <= waits:
                continue
            seen[j] = waits
            other, args = code[j]
            if other.startswith("v_mfma"):
                result, added = WAITS[other]
                if (waits < result and registers(args[0]) & (written | read)) or (waits < added and registers(args[3]) & written):
                    found.append((f"{name} {','.join(ops)}", f"{other} {','.join(args)}", waits))
            step = int(args[0], 0) + 1 if other == "s_nop" else 1
            ways += [(k, waits + step) for k in before[j]]
    return sum(name.startswith("v_fma_mix") for name, _ in code), found


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="no disassembler")
def test_vector_instructions_wait_for_matrix_instructions(tmp_path):
    shutil.copy(ssam.binding.LIB_PATH, tmp_path / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", "lib.so"], cwd=tmp_path, check=True, capture_output=True)
    kernels = {}
    for obj in sorted(tmp_path.glob("lib.so.*gfx950")):
        if b"delta_" not in obj.read_bytes():
            continue
        text = subprocess.run([OBJDUMP, "-d", "--symbolize-operands", "--no-show-raw-insn", str(obj)], check=True, capture_output=True, text=True).stdout
        for part in re.split(r"\n(?=[0-9a-f]+ <_Z)", text):
            m = re.match(r"[0-9a-f]+ <(_Z\w*delta_\w+)>:", part)
            if m and "v_mfma" in part:
                kernels[m[1]] = part.split("\n")
    assert sum("delta_walk" in n for n in kernels) >= 12 and sum("delta_back" in n for n in kernels) >= 36, len(kernels)
    for name, lines in kernels.items():
        many, found = too_early(lines)
        assert (many > 30 or "prepare" in name) and not found, (name, many, len(found), found[:3])

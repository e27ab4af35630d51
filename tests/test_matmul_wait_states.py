"""The scaled matrix instructions of the tiled product of 8-bit matrices stand in inline assembly, where the compiler adds none of the
wait states that they need: read from the assembly of the kernel's own build that every one of them has its wait states all the same, that
its accumulators stay where they are, and that nothing of the kernel is in scratch memory."""
import os
import re
import subprocess

import pytest

from paper_2503_06823_amd import build as B
from test_mfma_wait_states import MFMA_TO_READ, VALU_TO_MFMA, operands, registers, wait_states


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    out = tmp_path_factory.mktemp("asm") / "kernel.s"
    subprocess.run([B._hipcc(), *B.FLAGS, "-S", "--cuda-device-only", os.path.join(B.CSRC, "matmul_f8_tiled.hip"), "-o", str(out)], check=True,
                   capture_output=True)
    found, lines, name = {}, None, None
    text = open(out).read()
    for line in text.splitlines():
        m = re.match(r"(_ZN4emoe\S*tiled_kernel\S*):", line)
        if m:
            name, lines = m.group(1), []
        elif line.startswith(".Lfunc_end") and lines is not None:
            found[name] = lines
            lines = None
        elif lines is not None:
            t = line.split(";")[0].strip() if "#ASM" not in line else line.strip().lstrip(";")
            if t and not t.startswith("."):
                lines.append(t)
    scratch = re.findall(r"\.name:\s+(\S*tiled_kernel\S*)\n.*?\.private_segment_fixed_size: (\d+)", text, re.S)
    assert len(found) == 3 and len(scratch) == 3
    return found, scratch


def test_nothing_is_in_scratch_memory(kernels):
    assert [k for k in kernels[1] if k[1] != "0"] == []


def test_operands_are_written_long_enough_before(kernels):
    for name, code in kernels[0].items():
        n = 0
        for i, text in enumerate(code):
            if not text.startswith("v_mfma"):
                continue
            n += 1
            ops = [o.split(" ")[0] for o in operands(text)]
            read = registers(ops[1], "v") | registers(ops[2], "v") | registers(ops[4], "v") | registers(ops[5], "v")
            assert len(read) == 18, text
            states, j = 0, i - 1
            while states < VALU_TO_MFMA and j >= 0:
                before = code[j]
                if before.startswith("v_") and not before.startswith(("v_mfma", "v_cmp", "v_readlane", "v_readfirstlane")):
                    written = registers(operands(before)[0], "v")
                    if before.startswith("v_permlane") or before.startswith("v_swap"):
                        written |= registers(operands(before)[1], "v")
                    assert not written & read, f"{name}: '{before}' {states} wait states before '{text}'"
                states += wait_states(before)
                j -= 1
        assert n >= 4 * 64, name


def test_accumulators_are_matrix_results_read_long_enough_after(kernels):
    for name, code in kernels[0].items():
        reads = 0
        for i, text in enumerate(code):
            if text.startswith("#") or not re.search(r"\ba(\d+|\[)", text):
                continue
            assert text.startswith(("v_mfma", "v_accvgpr_read", "v_accvgpr_write")), f"{name}: {text}"  # no copies, no loads, no spills
            if text.startswith("v_accvgpr"):
                reads += 1
                states, j = 0, i - 1
                while states < MFMA_TO_READ and j >= 0:
                    assert not code[j].startswith("v_mfma"), f"{name}: '{text}' {states} wait states after '{code[j]}'"
                    states += wait_states(code[j])
                    j -= 1
        assert reads >= 256, name

"""The tiled products that also note which elements of h lie near a tie of two codes: held to what test_matmul_wait_states.py asks of the others."""
import os
import re
import subprocess

import pytest

from paper_2503_06823_amd import build as B
# run here on this module's kernels
from test_matmul_wait_states import (test_accumulators_are_matrix_results_read_long_enough_after, test_nothing_is_in_scratch_memory,  # noqa: F401
                                     test_operands_are_written_long_enough_before)


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    out = tmp_path_factory.mktemp("asm") / "kernel.s"
    subprocess.run([B._hipcc(), *B.FLAGS, "-S", "--cuda-device-only", os.path.join(B.CSRC, "matmul_f8_ties.hip"), "-o", str(out)], check=True,
                   capture_output=True)
    found, lines, name = {}, None, None
    text = open(out).read()
    for line in text.splitlines():
        m = re.match(r"(_ZN4emoe\S*tiled_ties\S*):", line)
        if m:
            name, lines = m.group(1), []
        elif line.startswith(".Lfunc_end") and lines is not None:
            found[name] = lines
            lines = None
        elif lines is not None:
            t = line.split(";")[0].strip() if "#ASM" not in line else line.strip().lstrip(";")
            if t and not t.startswith("."):
                lines.append(t)
    scratch = re.findall(r"\.name:\s+(\S*(?:tiled_ties|near_ties_kernel)\S*)\n.*?\.private_segment_fixed_size: (\d+)", text, re.S)
    assert len(found) == 2 and len(scratch) == 4
    return found, scratch

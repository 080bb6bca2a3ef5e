"""What the built library says of the masked attention kernels: their row maxima are inline asm, in front of which the compiler
inserts no wait states, and 12 of them must lie between a matrix instruction of 8 passes and a reader of its result."""
import os
import re
import subprocess
import sys

import pytest

from paper_2604_04335_amd.build import LIB_PATH

sys.path.insert(0, os.path.dirname(__file__))
from test_kernel_resources import NOTE, OBJDUMP, _registers  # noqa: E402


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="no disassembler")
def test_masked_maxima_wait_for_their_scores(tmp_path):
    blob = open(LIB_PATH, "rb").read()
    starts = [m.start() for m in re.finditer(re.escape(b"\x7fELF"), blob)][1:]  # the first is the host library's own
    parts = [blob[at:starts[i + 1] if i + 1 < len(starts) else len(blob)] for i, at in enumerate(starts)]
    (code,) = [x for x in parts if b"masked_few_rows_kernel" in x and NOTE in x]
    (tmp_path / "code").write_bytes(code)
    text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", str(tmp_path / "code")], capture_output=True, text=True, check=True).stdout
    lines, checked = [x.split("//")[0].strip() for x in text.splitlines()], 0
    for i, line in enumerate(lines):
        if not line.startswith("v_mfma"):
            continue
        result = _registers(line.split(None, 1)[1].split(",")[0])
        now = 1  # wait states since it issued: one an instruction, n + 1 for s_nop n; the next of its kind issues 8 after the last
        last = 0
        for after in lines[i + 1:]:
            op, _, operands = after.partition(" ")
            if now > 12 or op in ("s_branch", "s_endpgm") or after.endswith(":"):
                break
            if op == "v_max3_f32":
                checked += 1
                sources = set().union(*(_registers(x.strip().strip("|")) for x in operands.split(",")[1:]))
                assert not result & sources, (line, after, now - 1)
            if op.startswith("v_mfma"):
                now = last = max(now, last + 8)
            now += int(operands) + 1 if op == "s_nop" else 1
    assert sum(x.startswith("v_max3_f32") for x in lines) > 100

"""The transfers from memory to LDS in the compiled products of linear_ce.hip, as in test_kv_wait_states."""
import os
import re
import subprocess

import pytest

from paper_2609_36601_amd import build
from tests.test_kv_wait_states import problems


@pytest.mark.parametrize("part", [0, 1, 2, 3])
def test_transfers_wait(part, tmp_path):
    out = str(tmp_path / "a.s")
    subprocess.run([build.hipcc(), *build.HIPCC_FLAGS, f"-DSAKI_PART={part}", "--cuda-device-only", "-S",
                    os.path.join(build.CSRC, "linear_ce.hip"), "-o", out], check=True, capture_output=True)
    text = open(out).read()
    found, n = problems(text)
    assert n > 0 and not found, found[:5]
    # what writes m0 puts it back
    for block in re.findall(r"#ASMSTART\n(.*?)#ASMEND", text, re.S):
        if "m0" in block:
            keep = re.search(r"s_mov_b32 (s\d+), m0", block)[1]
            assert block.split("\n")[-2].strip() == f"s_mov_b32 m0, {keep}"

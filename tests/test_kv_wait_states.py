"""The transfers from memory to LDS in the compiled attention kernels: m0 and the base's scalar registers have settled
when one is issued.  (They are written in inline assembly, in which the compiler looks for no hazards.)"""
import os
import re
import subprocess

import pytest

from paper_2609_36601_amd import build


def scalars(operand):
    m = re.fullmatch(r"s\[(\d+):(\d+)\]", operand)
    if m:
        return set(range(int(m[1]), int(m[2]) + 1))
    m = re.fullmatch(r"s(\d+)", operand)
    return {int(m[1])} if m else set()


def problems(text):
    """Transfers that are issued too early, among the instructions in their order, and their number."""
    m0, vector, clock, found, n = -10**6, {}, 0, [], 0  # when m0, and scalar registers by a vector instruction, were written
    for number, line in enumerate(text.splitlines(), 1):
        line = line.split(";")[0].strip()
        if not line or line.startswith(".") or line.endswith(":"):
            continue
        name, _, rest = line.partition(" ")
        args = [a.strip() for a in rest.split(",")]
        if name.startswith("global_load_lds"):
            n += 1
            base = scalars(args[1].split()[0])
            if clock - m0 < 2 or any(clock - vector.get(r, -10**6) < 6 for r in base):
                found.append((number, line))
        if name.startswith("s_nop"):
            clock += int(args[0], 0)
        elif args[0] == "m0":
            m0 = clock
        elif name.startswith("v_"):
            for a in args[:2]:
                vector.update({r: clock for r in scalars(a)})
        elif name.startswith("s_"):
            for r in scalars(args[0]):
                vector.pop(r, None)
        clock += 1
    return found, n


def test_the_check_itself():
    assert problems("s_mov_b32 m0, s1\nglobal_load_lds_dwordx4 v1, s[2:3]")[0]
    assert not problems("s_mov_b32 m0, s1\ns_nop 0\nglobal_load_lds_dwordx4 v1, s[2:3]")[0]
    late = "v_readlane_b32 s3, v1, 0\ns_mov_b32 m0, s1\ns_nop {}\nglobal_load_lds_dwordx4 v1, s[2:3]"
    assert problems(late.format(2))[0] and not problems(late.format(3))[0]
    assert not problems("v_readlane_b32 s3, v1, 0\ns_add_u32 s3, s3, s4\ns_mov_b32 m0, s1\ns_nop 0\n"
                        "global_load_lds_dwordx4 v1, s[2:3]")[0]


@pytest.mark.parametrize("part", [0, 1])
def test_transfers_wait(part, tmp_path):
    out = str(tmp_path / "a.s")
    subprocess.run([build.hipcc(), *build.HIPCC_FLAGS, f"-DSAKI_PART={part}", "--cuda-device-only", "-S",
                    os.path.join(build.CSRC, "kv_attention.hip"), "-o", out], check=True, capture_output=True)
    text = open(out).read()
    found, n = problems(text)
    assert n > 0 and not found, found[:5]
    # what writes m0 puts it back
    for block in re.findall(r"#ASMSTART\n(.*?)#ASMEND", text, re.S):
        if "m0" in block:
            keep = re.search(r"s_mov_b32 (s\d+), m0", block)[1]
            assert block.split("\n")[-2].strip() == f"s_mov_b32 m0, {keep}"

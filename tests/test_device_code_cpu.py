"""The compiled state-cache and parameter-list kernels, read as assembly (no
GPU): no conditional select or branch takes the carry flag of an addition for a
comparison's result.  This compiler has dropped the instruction that moves a
64-bit comparison into the flag where a value was both selected and branched on
by it; the select then used the carry of an unrelated address addition."""
import os
import re
import subprocess

import pytest

from paper_2508_06993_amd.build import COMMON_FLAGS, CSRC, DEVICE_FLAGS, hipcc

# what sets the flag (scalar arithmetic, logic and comparisons)
SETS = re.compile(r"s_(cmp|cmpk|bitcmp|and|or|xor|andn2|orn2|nand|nor|xnor|not|lshl|lshr|ashr|bfe|"
                  r"bcnt|wqm|quadmask|abs|absdiff|min|max|add|addk|addc|sub|subb)")
CARRY = re.compile(r"s_(add_u32|addc_u32|sub_u32|subb_u32)$")


def flags_misread(assembly):
    """Selects and branches on the flag whose last setter before them is an
    addition with carry, except its own use as a carry mask (selects of -1 and 0)."""
    bad, last = [], None
    for line in assembly.splitlines():
        line = line.split(";")[0].strip()
        if re.match(r"[^.\s]\S*:", line):
            last = None
        if not line.startswith("s_"):
            continue
        op = line.split()[0]
        if op.startswith(("s_cselect", "s_cbranch_scc", "s_cmov")):
            if last and CARRY.match(last) and not line.endswith("-1, 0"):
                bad.append((last, line))
        elif SETS.match(op):
            last = op
    return bad


def test_the_check_sees_the_pattern():
    wrong = "k:\n s_add_u32 s0, s1, s2\n s_addc_u32 s3, s4, s5\n s_cbranch_vccz .L\n" \
            " s_cselect_b32 s6, s7, 0x80\n"
    right = wrong.replace(" s_cselect", " s_and_b64 vcc, vcc, exec\n s_cselect")
    assert len(flags_misread(wrong)) == 1 and not flags_misread(right)
    assert not flags_misread("k:\n s_add_u32 s0, s1, s2\n s_cselect_b64 s[4:5], -1, 0\n")


@pytest.mark.parametrize("name", ["state_cache.hip", "params.hip"])
def test_no_flag_is_misread(name, tmp_path):
    out = str(tmp_path / "code.s")
    flags = [f for f in COMMON_FLAGS if f != "-fPIC"]
    subprocess.run([hipcc(), *flags, *DEVICE_FLAGS, "-S", "--cuda-device-only",
                    os.path.join(CSRC, name), "-o", out], check=True, capture_output=True)
    with open(out) as f:
        text = f.read()
    assert text.count("s_endpgm") > 5
    assert flags_misread(text) == []

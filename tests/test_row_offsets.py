"""Rows of logits through buffer resources, in the built library's assembly: a
resource ends with the row, and a load past that end reads nothing, because the
whole offset stands in the lane's register.  A part of it in a scalar register
is left out of the comparison with the resource's size, or subtracted from that
size, which may be the smaller."""
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PATH = os.path.join(ROOT, "paper_2403_11366_amd", "_build", "lora_logits-hip-amdgcn-amd-amdhsa-gfx950.s")
ACCESS = re.compile(r"buffer_(load|store)_(ubyte|sbyte|ushort|sshort|byte|short|dword)\w*$")


def scalar_offsets(lines):
    """(buffer accesses, those with an offset besides the lane's and the instruction's)"""
    seen, found = 0, []
    for line in lines:
        line = line.split(";")[0].strip()
        op, _, rest = line.replace("\t", " ").partition(" ")
        if not ACCESS.match(op):
            continue
        seen += 1
        if rest.split(",")[-1].split()[0] != "0":
            found.append(line)
    return seen, found


def test_offsets_are_found():
    lane, scalar = "\tbuffer_load_dwordx4 v[0:3], v9, s[4:7], 0 offen offset:16", "\tbuffer_load_dwordx4 v[0:3], v9, s[4:7], s2 offen"
    assert scalar_offsets([lane, "; buffer_load_dword", "\tbuffer_wbl2 sc1", "\tbuffer_store_short v1, v9, s[4:7], 0 offen"]) == (2, [])
    assert scalar_offsets([lane, scalar]) == (2, [scalar.strip()])


def test_row_accesses_have_no_scalar_offset():
    if not os.path.exists(PATH):
        pytest.skip("library not built here")
    with open(PATH) as f:
        seen, found = scalar_offsets(f.read().split("\n"))
    assert seen > 100
    assert found == [], (len(found), found[:3])

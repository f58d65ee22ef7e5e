"""Wide stores in the built library's assembly: the instruction right behind a
store of three or four registers must not write one of them.  With a part of the
offset in a scalar register the compiler leaves such a pair in place, and its new
value has been stored."""
import glob
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
STORE = re.compile(r"(buffer|global|flat|scratch)_store_dwordx[34]$")


def registers(text):
    m = re.match(r"v\[(\d+):(\d+)\]$", text)
    if m:
        return set(range(int(m[1]), int(m[2]) + 1))
    m = re.match(r"v(\d+)$", text)
    return {int(m[1])} if m else set()


def overwritten_stores(lines):
    found, data = [], set()
    for line in lines:
        line = line.split(";")[0].strip()
        if not line or line.startswith(".") or line.endswith(":"):
            continue
        op, _, rest = line.partition(" ") if " " in line else line.partition("\t")
        args = [a.strip() for a in rest.split(",")]
        if op.startswith("v_") and registers(args[0]) & data:
            found.append(line)
        data = set()
        if STORE.match(op):
            data = registers(args[0] if op.startswith("buffer") else args[1])
    return found


def test_pairs_are_found():
    store, write = "\tbuffer_store_dwordx4 v[26:29], v1, s[48:51], s96 offen", "\tv_mul_f32_e32 v26, v94, v107"
    assert overwritten_stores([store, "; note", write]) == [write.strip()]
    assert overwritten_stores([store, "\ts_nop 1", write]) == []
    assert overwritten_stores([store, "\tv_mul_f32_e32 v30, v26, v27"]) == []
    assert overwritten_stores(["\tglobal_store_dwordx4 v[0:1], v[4:7], off", "\tv_mov_b32_e32 v6, 0"]) != []
    assert overwritten_stores(["\tbuffer_store_dwordx2 v[4:5], v1, s[0:3], 0 offen", "\tv_mov_b32_e32 v4, 0"]) == []


def test_built_kernels_have_none():
    files = sorted(glob.glob(os.path.join(ROOT, "paper_2403_11366_amd", "_build", "*-hip-amdgcn-amd-amdhsa-gfx950.s")))
    if not files:
        pytest.skip("library not built here")
    stores = 0
    for path in files:
        with open(path) as f:
            lines = f.read().split("\n")
        stores += sum(bool(re.search(r"\w+_store_dwordx[34]\b", x)) for x in lines)
        assert overwritten_stores(lines) == [], path
    assert stores > 100

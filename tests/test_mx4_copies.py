"""What the tiles of the 4-bit linear layer copy: address by address on the host
(tests/sanitize/mx4_copies.cpp), and the loads of scales in the built assembly,
whose offsets stand in the lanes' registers.  No GPU is used."""
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PKG = os.path.join(ROOT, "paper_2403_11366_amd")
HOST_SAN = ["-O1", "-g", "-fno-sanitize-recover=all", "-std=c++17", "-Xarch_host", "-fsanitize=address,undefined"]


def test_copies_stay_inside_their_operands(tmp_path):
    from paper_2403_11366_amd import build
    exe = str(tmp_path / "mx4_copies")
    cmd = [build.hipcc()] + HOST_SAN + ["-I", os.path.join(ROOT, "include"), "-I", os.path.join(PKG, "csrc"),
                                        os.path.join(ROOT, "tests", "sanitize", "mx4_copies.cpp"), "-o", exe]
    made = subprocess.run(cmd, capture_output=True, text=True, timeout=300)
    assert made.returncode == 0, made.stderr
    # the HIP runtime's own allocations outlive main: leak checking off
    res = subprocess.run([exe], capture_output=True, text=True, timeout=300, env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0"))
    assert res.returncode == 0 and "outside 0" in res.stdout, res.stdout + res.stderr
    assert int(re.search(r"copies (\d+)", res.stdout)[1]) > 10 ** 6


def test_loads_of_scales_have_no_scalar_offset():
    path = os.path.join(PKG, "_build", "lora_mx4-hip-amdgcn-amd-amdhsa-gfx950.s")
    if not os.path.exists(path):
        pytest.skip("library not built here")
    with open(path) as f:
        loads = [x.split(";")[0].strip() for x in f if "buffer_load_dwordx2" in x]
    assert loads and all(x.split(",")[-1].split()[0] == "0" for x in loads), loads

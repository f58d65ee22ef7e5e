"""The C ABI of the operators around the layer's output under the host sanitizers
(tests/sanitize/ops_sanitize.cpp: refusals, and what each kernel assumes of the
shapes that its launch rule gives it), and the GPU tests' sizes against the
kernels of the 4-bit forward: all of them are reached.  No GPU is used."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PKG = os.path.join(ROOT, "paper_2403_11366_amd")
HOST_SAN = ["-O1", "-g", "-fno-sanitize-recover=all", "-fno-omit-frame-pointer", "-std=c++17"]
SAN = ["-Xarch_host", "-fsanitize=address,undefined"]


def _run(cmd, **kw):
    res = subprocess.run(cmd, capture_output=True, text=True, timeout=300, **kw)
    assert res.returncode == 0, f"{' '.join(cmd)}\n{res.stdout}\n{res.stderr}"
    return res.stdout


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    from paper_2403_11366_amd import build
    objs = [os.path.join(build.BUILD, s + ".o") for s in build.SOURCES if s.endswith(".hip")]
    if not all(os.path.exists(o) for o in objs):
        build.build()
    out = tmp_path_factory.mktemp("ops_san")
    inc = ["-I", os.path.join(ROOT, "include"), "-I", os.path.join(PKG, "csrc")]
    made = []
    for src in (os.path.join(PKG, "csrc", "lora_ops_abi.cpp"), os.path.join(ROOT, "tests", "sanitize", "ops_sanitize.cpp")):
        made.append(str(out / (os.path.basename(src) + ".o")))
        _run([build.hipcc()] + HOST_SAN + SAN + inc + ["-c", src, "-o", made[-1]])
    exe = str(out / "ops_san")
    _run([build.hipcc()] + SAN + made + objs + ["-o", exe])
    return exe


def test_refusals_and_plans_under_sanitizers(driver):
    # the HIP runtime's own allocations outlive main: leak checking off
    text = _run([driver], env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0", UBSAN_OPTIONS="print_stacktrace=1"))
    assert "driver: ok" in text and int(text.split("plans checked:")[1]) > 10000


def test_gpu_sizes_reach_every_kernel_of_the_4_bit_forward(driver):
    import test_gpu_mx4 as gpu
    import test_gpu_mx4_kernels as kernels
    sizes = [str(x) for shape in gpu.LINEAR + kernels.SIZES for x in shape]
    text = _run([driver] + sizes, env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0"))
    assert set(text.split()) == {str(i) for i in range(9)}

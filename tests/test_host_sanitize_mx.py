"""Host sanitizer build of the 4-bit cache's and the adjustment's host side (target_mx_abi.cpp), as
test_host_sanitize_target.py does for the other target-side calls.  No GPU and no HIP runtime are involved."""
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CXX = "/opt/rocm/llvm/bin/clang++"
CSRC = os.path.join(ROOT, "paper_2609_24197_amd", "csrc")
ABI = os.path.join(CSRC, "target_mx_abi.cpp")

pytestmark = pytest.mark.skipif(not os.path.exists(CXX), reason="ROCm clang++ not installed")


def _build(abi: str, out: str) -> None:
    cmd = [CXX, "-std=c++20", "-O1", "-g", "-fno-omit-frame-pointer", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
           f"-I{ROOT}/include", f"-I{CSRC}", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", abi,
           os.path.join(CSRC, "target_abi.cpp"), os.path.join(ROOT, "tests", "host_sanitize", "mx_driver.cpp"), "-o", out]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-4000:]


def _run(exe: str):
    return subprocess.run([exe], capture_output=True, text=True, timeout=300,
                          env=dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0"))


def test_clean_under_asan_ubsan(tmp_path):
    exe = str(tmp_path / "mx")
    _build(ABI, exe)
    r = _run(exe)
    assert r.returncode == 0, (r.stdout[-2000:], r.stderr[-4000:])
    m = re.search(r"(\d+) cases passed", r.stdout)
    assert m and int(m.group(1)) >= 2800, r.stdout[-2000:]


@pytest.mark.parametrize("good,bad", [("a.part_ml = ar.take<float>(rows * 2);", "a.part_ml = ar.take<float>(rows);"),
                                      ("a.flags = ar.take<int>(a.max_flags);", "a.flags = ar.take<int>(a.max_flags / 8);")])
def test_a_region_cut_too_small_is_caught(tmp_path, good, bad):
    src = open(ABI).read()
    assert good in src
    abi = tmp_path / "target_mx_abi.cpp"
    abi.write_text(src.replace(good, bad))
    exe = str(tmp_path / "mx_bad")
    _build(str(abi), exe)
    assert _run(exe).returncode != 0

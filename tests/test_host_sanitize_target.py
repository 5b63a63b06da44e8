"""Host sanitizer build of the target-side entry points' host side (target_abi.cpp), as test_host_sanitize.py does for
the drafting calls: argument checks, workspace regions and extents, and the attention plan's arithmetic, on the CPU
under AddressSanitizer and UndefinedBehaviorSanitizer.  No GPU and no HIP runtime are involved."""
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CXX = "/opt/rocm/llvm/bin/clang++"
ABI = os.path.join(ROOT, "paper_2609_24197_amd", "csrc", "target_abi.cpp")

pytestmark = pytest.mark.skipif(not os.path.exists(CXX), reason="ROCm clang++ not installed")


def _build(abi: str, out: str) -> None:
    cmd = [CXX, "-std=c++20", "-O1", "-g", "-fno-omit-frame-pointer", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
           f"-I{ROOT}/include", f"-I{ROOT}/paper_2609_24197_amd/csrc", "-fsanitize=address,undefined",
           "-fno-sanitize-recover=all", abi, os.path.join(ROOT, "tests", "host_sanitize", "target_driver.cpp"), "-o", out]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-4000:]


def _run(exe: str):
    return subprocess.run([exe], capture_output=True, text=True, timeout=300,
                          env=dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0"))


def test_clean_under_asan_ubsan(tmp_path):
    exe = str(tmp_path / "target")
    _build(ABI, exe)
    r = _run(exe)
    assert r.returncode == 0, (r.stdout[-2000:], r.stderr[-4000:])
    m = re.search(r"(\d+) cases passed", r.stdout)
    assert m and int(m.group(1)) > 4000, r.stdout[-2000:]


@pytest.mark.parametrize("good,bad", [("a.part_ml = ar.take<float>(rows * 2);", "a.part_ml = ar.take<float>(rows);"),
                                      ("a.units = ar.take<hspec::ChunkUnit>(a.max_units);",
                                       "a.units = ar.take<hspec::ChunkUnit>(a.max_units / 2);")])
def test_a_region_cut_too_small_is_caught(tmp_path, good, bad):
    src = open(ABI).read()
    assert good in src
    abi = tmp_path / "target_abi.cpp"
    abi.write_text(src.replace(good, bad))
    exe = str(tmp_path / "target_bad")
    _build(str(abi), exe)
    assert _run(exe).returncode != 0
